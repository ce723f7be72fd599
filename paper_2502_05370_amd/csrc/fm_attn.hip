// Attention of one new token per slot over the pages of its sequence.
//
// A wavefront takes a step of 16 to 128 tokens of a key head at a time, 8 KB of keys
// or more, for up to 16 query heads that read it.  The pages hold operands: a piece
// of 1 KB is one load of 16 bytes a lane, whole lines, and the very registers that
// the matrix instructions take.
//   scores   S^T = K Q^T: rows are tokens, columns are queries.  Lane 16 g + c gets
//            tokens 4 g .. 4 g + 3 of each block of 16, for query c.
//   output   O^T += V^T P^T: the same lane must hold P of query c for four tokens
//            per block, which are the ones it has, so that the probabilities pass
//            from accumulators to operands without changing lanes.
// Running maximum and sum per query; the sums and outputs are scaled only when a
// maximum has grown.
//
// Memory bounds long batches: with bf16, 16 queries per key head cost the matrix units
// 7% of the time that the keys and values take to arrive (float32, whose instructions
// are a tenth as fast, a third).  One request of 131,072 tokens, 32 query heads on 8 of
// 128: 537 MB stream in 77 us (7.0 TB/s) of 88 for the call; 64 requests of 1 to
// 8,192 tokens: 1.02 GB in 160 us.  Short batches are bound by a chain of waits:
// lengths, table, keys, joins; three requests of 37 tokens take 7.9 us, one of 4,096
// tokens 14.
#include "fm_device.h"
#include "fm_kv.h"
#include "fm_mma.h"

namespace fm {

namespace {

constexpr int kAttnWaves = 4;   // wavefronts of a workgroup
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

// What p cut to `cut` leaves: at least the least bf16 above zero, or nothing where p is
// zero (NaN stays NaN in the cut part).  The median, since 0 <= p - cut <= p.
__device__ __forceinline__ float rest(float p, uint32_t cut) {
  return __builtin_amdgcn_fmed3f(p - __uint_as_float(cut), p, 0x1p-133f);
}

// The tokens that a slot's query sees.
struct Seen {
  int32_t lo, hi;   // places
  __device__ __forceinline__ bool none() const { return lo >= hi; }
};
__device__ __forceinline__ Seen seen_of(const AttnArgs& a, int s) {
  const int32_t len = a.c.tokens(a.c.length[s]);
  // (a null array's place is taken by the lengths, and what is read there not used)
  const int32_t from = (a.first != nullptr ? a.first : a.c.length)[s];
  const uint8_t on = a.active != nullptr ? a.active[s] : 1;
  int32_t lo = a.first != nullptr && from > 0 ? from : 0;
  if (a.window > 0 && len - a.window > lo) lo = len - a.window;
  if (on == 0) lo = len;
  return Seen{lo, len};
}

// ALONE: no other workgroup reads these keys.
template <typename T, int NP, bool ALONE>
struct Wave {
  static constexpr bool kBf = sizeof(T) == 2;
  // Blocks of a step: 8 KB of keys or more (bf16 takes blocks in pairs), so that a
  // CU's four wavefronts have 64 KB and more on their way.
  static constexpr int SB = NP >= 8 ? (kBf ? 2 : 1) : (NP >= 4 ? 2 : (NP == 1 ? 8 : 4));
  static constexpr int OT = NP * (kBf ? 2 : 1);   // tiles of 16 dimensions
  static constexpr bool kTwo = NP <= (kBf ? 5 : 9);   // registers for two workgroups per CU
  // Rows so short that weighing a step takes longer than loading it: a second workgroup
  // fills the time (64 slots of 2,048 tokens, 8 heads of 32 bf16: 47 us and 36; of 64
  // float32: 106 and 95; heads of 64 bf16, 4,096 tokens: 96 and 93).
  static constexpr bool kNarrow = NP <= (kBf ? 2 : 4);
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
  // What no other workgroup reads passes the caches by: with 32 query heads on 8, 64
  // requests of 1 to 8,192 tokens 160 us, 181 through them; with 24 on each of 4, 127
  // past them and 120 through them.
  static __device__ __forceinline__ void load(const char* at, uint32x4 (&r)[NP]) {
    const uint32x4* p = reinterpret_cast<const uint32x4*>(at) + threadIdx.x % kWave;
#pragma unroll
    for (int t = 0; t < NP; ++t) {
      if constexpr (ALONE) r[t] = __builtin_nontemporal_load(p + t * (kPieceBytes / 16));
      else r[t] = p[t * (kPieceBytes / 16)];
    }
  }
  __device__ __forceinline__ void scores(floatx4 (&s)[SB]) const {
#pragma unroll
    for (int b = 0; b < SB; ++b) {
      s[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < NP; ++t) s[b] = mma_step<T>(k[b][t], q[t], s[b]);
    }
  }
  // Tokens of block b outside [lo[b], hi[b]) have no part, nor have their values.
  __device__ __forceinline__ void mask(floatx4 (&s)[SB], const int (&lo)[SB], const int (&hi)[SB]) {
    const int row = threadIdx.x % kWave / 16 * 4;
#pragma unroll
    for (int b = 0; b < SB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const bool in = row + r >= lo[b] && row + r < hi[b];
        s[b][r] = in ? s[b][r] : -__builtin_inff();
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
  // Scores (as powers of two) to weights, in place.
  __device__ __forceinline__ void weigh(floatx4 (&s)[SB]) {
    float top = -__builtin_inff();
#pragma unroll
    for (int b = 0; b < SB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, s[b][r]);
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
        s[b][r] = __builtin_amdgcn_exp2f(s[b][r] - base);
        l += s[b][r];
      }
  }
  __device__ __forceinline__ void add(const floatx4 (&p)[SB]) {
    if constexpr (kBf) {
      // p as two bf16, so that the result is off by its own rounding alone: p cut
      // towards zero, and the rest.  2^-133 stands for a rest of zero, so that an
      // infinite value gives infinity and not the NaN of infinity times zero; a weight of
      // zero is zero in both parts.
      uint32x4 hi, lo;
#pragma unroll
      for (int b = 0; b < SB; b += 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = p[b + i / 2][i % 2 * 2], y = p[b + i / 2][i % 2 * 2 + 1];
          hi[i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
          lo[i] = pack_bf16(rest(x, hi[i] << 16), rest(y, hi[i] & 0xFFFF0000u));
        }
#pragma unroll
        for (int t = 0; t < NP; ++t)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32x4 w = {v[b][t][2 * i], v[b][t][2 * i + 1], v[b + 1][t][2 * i], v[b + 1][t][2 * i + 1]};
            o[2 * t + i] = mma_step<T>(w, hi, o[2 * t + i]);
            o[2 * t + i] = mma_step<T>(w, lo, o[2 * t + i]);
          }
      }
    } else {
#pragma unroll
      for (int b = 0; b < SB; ++b)
#pragma unroll
        for (int t = 0; t < NP; ++t) o[t] = mma_step<T>(v[b][t], __builtin_bit_cast(uint32x4, p[b]), o[t]);
    }
  }
};

// Page numbers of a slot, one per lane: of its table's entries from `base` on.
struct Known {
  int base, ids;
  __device__ __forceinline__ void take(const AttnArgs& a, int slot, int entry) {
    const int mine = entry + static_cast<int>(threadIdx.x % kWave);
    base = entry;
    ids = a.c.table[static_cast<int64_t>(slot) * a.c.max_pages + (mine < a.c.max_pages ? mine : a.c.max_pages - 1)];
  }
  // of the first visible token on: sent for as soon as the slot is known
  __device__ __forceinline__ void begin(const AttnArgs& a, int slot, Seen seen) {
    if (!seen.none()) take(a, slot, entry_of(a, seen.lo / kBlockTokens));
  }
  static __device__ __forceinline__ int entry_of(const AttnArgs& a, int block) {
    return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(block)) * a.per_page_inv) >> 32);
  }
};

// A wavefront's steps [first, last) with a stride of a slot's blocks, counted from
// the block of the first visible token.
template <typename T, int NP, bool ALONE>
__device__ __forceinline__ void walk(const AttnArgs& a, Wave<T, NP, ALONE>& w, int slot, int head, Seen seen, Known& known,
                                     int first, int last, int stride, uint32_t& bad) {
  using W = Wave<T, NP, ALONE>;
  constexpr int SB = W::SB;
  const int per_page = a.c.page / kBlockTokens;
  const int block_bytes = NP * kPieceBytes;
  const char* keys = a.c.pages + a.c.head_offset(a.layer, 0, head);
  const int64_t to_values = a.c.head_offset(0, 1, 0);
  // (through an instruction of its own: a plain load next to a vector product is
  // widened over its neighbours, which puts those into scratch memory)
  const float scale2 = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(a.scale2)));
  const int b0 = seen.lo / kBlockTokens;
  const int b1 = (seen.hi + kBlockTokens - 1) / kBlockTokens;

  // where block b lies, and which of its tokens are seen: none of one that does
  // not exist or whose page does not, which stands at another's place
  auto locate = [&](int step, const char* (&at)[SB], int (&lo)[SB], int (&hi)[SB]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < SB; ++i) {
      const int b = b0 + step * SB + i;
      const int bb = b < b1 ? b : b1 - 1;
      const int entry = Known::entry_of(a, bb);
      if (entry < known.base || entry >= known.base + kWave) known.take(a, slot, entry);
      int page = __builtin_amdgcn_readlane(known.ids, entry - known.base);
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
  // Keys are sent for when the step before has used its own, values likewise.  The
  // first turn only sends: one copy of the code, which comes from memory when the
  // caches hold keys.
  const char* at[SB];
  int lo[SB], hi[SB], lo0[SB], hi0[SB];
  floatx4 s[SB];
  bool have = false;
  for (int step = first;; step += stride) {
    const bool more = step < last;
    if (!(have || more)) break;
    if (have) {
      w.scores(s);
#pragma unroll
      for (int i = 0; i < SB; ++i) {
        s[i] *= scale2;
        lo0[i] = lo[i];
        hi0[i] = hi[i];
      }
    }
    if (more) {
      locate(step, at, lo, hi);
#pragma unroll
      for (int i = 0; i < SB; ++i) W::load(at[i], w.k[i]);
    }
    if (have) {
      bool whole = true;
#pragma unroll
      for (int i = 0; i < SB; ++i) whole = whole && lo0[i] <= 0 && hi0[i] >= kBlockTokens;
      if (!whole) w.mask(s, lo0, hi0);
      w.weigh(s);
      w.add(s);
    }
    if (more) {
#pragma unroll
      for (int i = 0; i < SB; ++i) W::load(at[i] + to_values, w.v[i]);
    }
    have = more;
  }
}

// Queries of a tile of one key head: lane 16 g + c holds 16 bytes of query c per 64.
template <typename T, int NP, bool ALONE>
__device__ __forceinline__ void load_queries(const AttnArgs& a, Wave<T, NP, ALONE>& w, int slot, int head, int query0) {
  constexpr int N = 16 / static_cast<int>(sizeof(T));
  const int lane = threadIdx.x % kWave;
  const int c = lane % 16 + query0, g = lane / 16;
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
template <int DIMS>   // of a padded row
struct Joined {
  static constexpr int kLd = DIMS + 4;
  float m[kAttnWaves][16], l[kAttnWaves][16];
  float o[kAttnWaves][16][kLd];
};

// A part in the workspace: m [16], l [16], outputs [queries of a tile][padded row].
__host__ __device__ inline uint32_t part_bytes(int32_t group, int dims) {
  return static_cast<uint32_t>(32 + (group < 16 ? group : 16) * dims) * sizeof(float);
}
// Parts are written and read past the caches of the XCDs (SC1, the bit of accesses
// of agent scope), 16 bytes a lane.
constexpr int kAgent = 16;

// How much of a part counts in a sum relative to the maximum `top`.  A part that saw
// no score has the maximum minus infinity, and one that saw only NaN too.
__device__ __forceinline__ float share(float m, float l, float top) {
  return m == -__builtin_inff() ? (l == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f(m - top);
}

// Query qi's maximum over the entries of `sh`, and their sum relative to it.
template <int DIMS>
__device__ __forceinline__ float total_of(const Joined<DIMS>& sh, int qi, float (&f)[kAttnWaves], float& top) {
  top = -__builtin_inff();
#pragma unroll
  for (int u = 0; u < kAttnWaves; ++u) top = fmaxf(top, sh.m[u][qi]);
  float all = 0.0f;
#pragma unroll
  for (int u = 0; u < kAttnWaves; ++u) {
    f[u] = share(sh.m[u][qi], sh.l[u][qi], top);
    all += f[u] * sh.l[u][qi];
  }
  return all;
}

// The entries of `sh` together, to the output.
template <typename T, int DIMS>
__device__ __forceinline__ void finish(const AttnArgs& a, const Joined<DIMS>& sh, int row0, int queries) {
  for (int i = threadIdx.x; i < queries * (DIMS / 4); i += kAttnWaves * kWave) {
    const int qi = i / (DIMS / 4), d = i % (DIMS / 4) * 4;
    if (d >= a.c.head_dim) continue;
    float f[kAttnWaves], top;
    const float all = total_of(sh, qi, f, top);
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < kAttnWaves; ++u) sum += f[u] * *reinterpret_cast<const floatx4*>(&sh.o[u][qi][d]);
    const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
    store4<T>(a.out, static_cast<int64_t>(row0 + qi) * a.c.head_dim + d, all == 0.0f ? zero : sum / all);
    if (d == 0 && a.lse != nullptr)
      a.lse[row0 + qi] = all == 0.0f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(all)) * kLn2;
  }
}

// The entries of `sh` together, as a part.
template <int DIMS>
__device__ __forceinline__ void store_part(const Joined<DIMS>& sh, int queries, __amdgpu_buffer_rsrc_t rs,
                                           uint32_t part) {
  for (int i = threadIdx.x; i < queries * (DIMS / 4); i += kAttnWaves * kWave) {
    const int qi = i / (DIMS / 4), d = i % (DIMS / 4) * 4;
    float f[kAttnWaves], top;
    const float all = total_of(sh, qi, f, top);
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < kAttnWaves; ++u) sum += f[u] * *reinterpret_cast<const floatx4*>(&sh.o[u][qi][d]);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint32x4, sum), rs, static_cast<int>(part + 128u + 16u * i),
                                           0, kAgent);
    if (d == 0) {
      __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(top), rs, static_cast<int>(part + 4u * qi), 0, kAgent);
      __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(all), rs, static_cast<int>(part + 64u + 4u * qi), 0, kAgent);
    }
  }
}

// n parts of a tile (part(i) their offsets) into `sh`, a wavefront every fourth of
// them: 4 U parts at a time, whose values are on their way while their maxima and
// sums decide how much each counts.
constexpr int kTurn = 32;   // parts at most
// Parts up to which more of each are on their way instead: 291 tokens, 16 queries on 2
// heads of 256 bf16 19.0 us in turns of 32 parts, 16.4 in turns of 8; 7 slots of 177, 48
// on 2, 24.4 and 19.1.  (A third form for 16 parts: 28.5 us -> 25.0 at 2,000 tokens on
// one head of 256 float32, but its code costs every call of 128 bf16 0.1-4 us.)
constexpr int kFewParts = 8;
struct Weights {
  float top[4 * kAttnWaves][16];   // by group of threads and query
  float scale[16];         // of what is there already
  float f[kTurn][16];
};
template <int U, int DIMS, typename Part>
__device__ __forceinline__ void collect(Joined<DIMS>& sh, Weights& wt, int queries, int n, __amdgpu_buffer_rsrc_t rs,
                                        Part part) {
  constexpr int kTurn = U * kAttnWaves;
  constexpr int G = 4 * kAttnWaves, J = (kTurn + G - 1) / G;   // groups of 16 threads, and parts whose weights each computes
  constexpr int E = 16 / U;               // fours of values of a lane in flight, per part
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int pg = tid / 16, pq = tid % 16;   // weights: parts pg + G j of a turn, query pq
  const int quads = queries * (DIMS / 4);
  float l = 0.0f, top = -__builtin_inff();   // of query pq; l: this thread's parts
  for (int p0 = 0; p0 < n; p0 += kTurn) {
    float m[J], s[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int p = p0 + pg + G * j;
      const bool in = pg + G * j < kTurn && p < n && pq < queries;
      const uint32_t at = in ? part(p) + 4u * pq : kOutside;
      m[j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, static_cast<int>(at), 0, kAgent));
      s[j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, static_cast<int>(in ? at + 64u : at), 0, kAgent));
      if (!in) m[j] = -__builtin_inff();
    }
    for (int e0 = 0; e0 < quads; e0 += E * kWave) {
      uint32x4 x[U][E];   // zeros past the parts and past their rows
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int p = p0 + wv + u * kAttnWaves;
        const uint32_t at = part(p < n ? p : n - 1) + 128u + 16u * (e0 + lane);
#pragma unroll
        for (int e = 0; e < E; ++e)
          x[u][e] = __builtin_amdgcn_raw_buffer_load_b128(
              rs, static_cast<int>(p < n && e0 + e * kWave + lane < quads ? at + e * (16u * kWave) : kOutside), 0, kAgent);
      }
      if (e0 == 0) {
        wt.top[pg][pq] = fmaxf(m[0], m[J - 1]);
        __syncthreads();
        float now = top;
#pragma unroll
        for (int j = 0; j < G; ++j) now = fmaxf(now, wt.top[j][pq]);
        l *= share(top, l, now);
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const float f = share(m[j], s[j], now);
          if (pg + G * j < kTurn) wt.f[pg + G * j][pq] = f;
          l += f * s[j];
        }
        if (pg == 0) wt.scale[pq] = top == now ? 1.0f : share(top, 1.0f, now);
        top = now;
        __syncthreads();
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = e0 + e * kWave + lane;
        if (i >= quads) continue;
        const int qi = i / (DIMS / 4), d = i % (DIMS / 4) * 4;
        floatx4* to = reinterpret_cast<floatx4*>(&sh.o[wv][qi][d]);
        floatx4 sum = {0.f, 0.f, 0.f, 0.f};
        if (p0 > 0) sum = *to * wt.scale[qi];
#pragma unroll
        for (int u = 0; u < U; ++u) sum += wt.f[wv + u * kAttnWaves][qi] * __builtin_bit_cast(floatx4, x[u][e]);
        *to = sum;
      }
    }
    __syncthreads();
  }
  wt.top[pg][pq] = l;
  __syncthreads();
  if (pg < kAttnWaves) {
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += wt.top[pg * 4 + j][pq];
    sh.m[pg][pq] = top;
    sh.l[pg][pq] = sum;
  }
  __syncthreads();
}

// n / d rounded down, d > 0, |n / d| < 2^20, without the long code of a division.
__device__ __forceinline__ int ratio(int n, int d) {
  int q = static_cast<int>(static_cast<float>(n) / static_cast<float>(d));
  while (static_cast<int64_t>(q) * d > n) --q;
  while (static_cast<int64_t>(q + 1) * d <= n) ++q;
  return q;
}

// The batch's work is a line: slot after slot, in it key head after key head, in it
// kOverhead units and one per step.  Every workgroup takes as much of the line,
// whatever the lengths are.  What it has of a tile, the 16 queries of a key head, is a
// part; a tile of several workgroups is joined by the last of them that is done
// (tickets, no wait), in the order of the line.  No part is shorter than kPart steps: a
// cut closer to an end of its tile moves there.
//
// More than 16 queries of a key head are tiles side by side: a piece of the line is
// taken by a workgroup for each, on one XCD, so that the keys that the first brings are
// in its L2 for the others: 64 requests of 1 to 8,192 tokens, 24 queries on each of 4
// bf16 heads of 128 or 256, 120 or 216 us.  One tile behind the other, which reads the
// keys from memory again, 169 or 321.  (A dropped form with both tiles in one
// wavefront's registers took 0.9 or 1.1 of the time side by side, but float32 heads of
// 256 spilled to twice it, and 8 requests of 1,000 tokens took 25 us for 19.)  More
// than kSide tiles take turns: 128 queries on one head of 128 79 us, 300 155.
//
// One workgroup per CU does for long tiles, whose parts it has few of to join: 64
// requests of 1 to 8,192 tokens 160 us, with two 167; one of 131,072 88 and 93.
// Where there are more tiles than CUs and they are short, each is a wait for its data
// and two per CU pay: 64 slots of 8 heads of 128 bf16, mean lengths of 128 / 512 /
// 1,024 / 2,048 tokens: one 19.1 / 38.4 / 53.5 / 91.6 us, two 15.6 / 34.8 / 52.0 / 93.6
// (kShort lies between the last two).  Workgroups side by side are two per CU where
// registers allow it, so that as many bytes are on their way: 64 requests of 1 to 8,192
// tokens, 24 queries on each of 4 heads of 128 bf16: one 152 us, two 120.
constexpr int kCus = 256;
constexpr int kWorkers = 2 * kCus;   // workgroups that the line is cut for at most
constexpr int kShort = 64;           // units of a tile on average
// Units of a tile besides its steps: three requests of 37 tokens 10.7 us with 4, 7.9
// with 8 and 12; 64 requests as above 160 with 4 and 8, 162 with 12; with a window of
// 1,000 (kPart) 22.6, 24.0 and 24.1.
constexpr int kOverhead = 8;
// Units of a workgroup at least, so that few tiles have a workgroup each and long ones
// are cut fine: one request of 2,160 tokens on one key head 13.4 us with 8, 15.6 with
// 16, 19.1 with 24.
constexpr int kLeast = 8;
constexpr int kSide = 8;             // tiles side by side
constexpr int kXcds = 8;             // that take workgroups in turn
// Steps of a part at least: 23 requests of 3,000 tokens with a window of 1,000, heads of
// 80 float32, 26.8 us with 8 and 24.0 with 4, but 7 slots of 177 as above 15.0 and 19.1.
constexpr int kPart = 4;
// Steps up to which a tile that shares a piece is a wavefront's alone: 103 slots of 4
// tokens, 32 heads of 128 bf16: 16 us, 34 without; 225 of 2, 3 heads of 256: 12 and 22.
constexpr int kFew = 4;
__device__ __forceinline__ int cut(int x, int steps) {   // x: from the tile's first step on
  if (x <= 0) return 0;
  if (x >= steps) return steps;
  return x < kPart ? 0 : (x > steps - kPart ? steps : x);
}

struct Sides {
  int32_t turns, side;   // tiles of a key head: turns x side or a few less
  int32_t pieces;        // that the line is cut into at most, of which `side` workgroups take each
};
Sides sides_of(int32_t group) {
  const int32_t tiles = (group + 15) / 16;
  const int32_t turns = (tiles + kSide - 1) / kSide;
  const int32_t side = (tiles + turns - 1) / turns;
  return Sides{turns, side, kWorkers / side / kXcds * kXcds};
}

template <typename T, int NP, bool ALONE>
__global__ void __launch_bounds__(kAttnWaves * kWave, (Wave<T, NP, ALONE>::kTwo ? 2 : 1))
    k_attn(AttnArgs a, Sides sides_given, uint32_t* tickets, char* parts, uint32_t parts_bytes) {
  using W = Wave<T, NP, ALONE>;
  constexpr int kDims = NP * kRowPiece / static_cast<int>(sizeof(T));
  constexpr int NT = kAttnWaves * kWave;
  __shared__ Joined<kDims> sh;
  __shared__ Weights weights;
  __shared__ int64_t sums[kAttnWaves];
  __shared__ int64_t where[2];
  __shared__ Seen begin;
  __shared__ int32_t is_last;
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int c = lane % 16, g = lane / 16;
  const Sides sides = ALONE ? Sides{1, 1, kWorkers} : sides_given;
  const int per_slot = a.c.heads * sides.turns;
  const int piece =
      static_cast<int>(ALONE ? blockIdx.x : blockIdx.x / (kXcds * sides.side) * kXcds + blockIdx.x % kXcds);
  const int beside = static_cast<int>(ALONE ? 0 : blockIdx.x / kXcds % sides.side);
  auto steps_of = [&](Seen w) __attribute__((always_inline)) {
    const int blocks = w.none() ? 0 : (w.hi + kBlockTokens - 1) / kBlockTokens - w.lo / kBlockTokens;
    return (blocks + W::SB - 1) / W::SB;
  };

  // First pass: the line's length.  Second pass: the slot in which this workgroup's
  // piece of it begins (slots that one round holds are not summed again).
  int64_t from = 0;   // the piece: `mine` units from there on
  int each = 0, mine = 0;
  for (int pass = 0; pass < 2; ++pass) {
    int64_t passed = 0, cost = 0, before = 0;
    Seen own{0, 0};
    auto begins_here = [&](int s) __attribute__((always_inline)) {
      if (from >= before && from < before + cost) {
        where[0] = s;
        where[1] = before - from;
        begin = own;
      }
    };
    for (int s0 = 0; s0 < a.c.n_slots; s0 += NT) {
      cost = 0;
      if (s0 + tid < a.c.n_slots) {
        own = seen_of(a, s0 + tid);
        cost = static_cast<int64_t>(per_slot) * (kOverhead + steps_of(own));
      }
      int64_t upto = cost;
#pragma unroll
      for (int m = 1; m < kWave; m <<= 1) {
        const int64_t o = __shfl_up(upto, m, kWave);
        if (lane >= m) upto += o;
      }
      __syncthreads();
      if (lane == kWave - 1) sums[wv] = upto;
      __syncthreads();
      before = passed + upto - cost;
#pragma unroll
      for (int w = 0; w < kAttnWaves; ++w) {
        before += w < wv ? sums[w] : 0;
        passed += sums[w];
      }
      if (pass == 1) begins_here(s0 + tid);
      if (pass == 1 && passed > from) break;
    }
    if (pass == 1) break;
    // One workgroup per CU, or two: where short tiles, more than CUs, each wait for
    // their data.
    const int64_t tiles = static_cast<int64_t>(a.c.n_slots) * per_slot;
    const bool two = W::kTwo && (W::kNarrow || !ALONE || (tiles > kCus && passed < kShort * tiles));
    each = static_cast<int>((passed + sides.pieces - 1) / sides.pieces) * (two ? 1 : 2);
    if (each < kLeast) each = kLeast;
    from = static_cast<int64_t>(each) * piece;
    if (from >= passed) return;
    mine = passed - from < each ? static_cast<int>(passed - from) : each;
    if (a.c.n_slots <= NT) {
      begins_here(tid);
      break;
    }
  }
  __syncthreads();
  int slot = __builtin_amdgcn_readfirstlane(static_cast<int>(where[0]));
  uint32_t bad = 0;
  Seen seen = begin;
  Known known;
  known.begin(a, slot, seen);
  int steps = __builtin_amdgcn_readfirstlane(steps_of(seen));
  // the tile that the piece begins in, and where it begins itself: places are
  // counted from the piece's begin
  const int64_t back = -where[1];
  int tile0 = static_cast<int>(static_cast<float>(back) / static_cast<float>(kOverhead + steps));
  while (static_cast<int64_t>(tile0) * (kOverhead + steps) > back) --tile0;
  while (static_cast<int64_t>(tile0 + 1) * (kOverhead + steps) <= back) ++tile0;
  tile0 = __builtin_amdgcn_readfirstlane(tile0);
  int at = __builtin_amdgcn_readfirstlane(
      static_cast<int>(static_cast<int64_t>(tile0) * (kOverhead + steps) - back));
  int head = tile0 / sides.turns, round = tile0 % sides.turns;
  mine = __builtin_amdgcn_readfirstlane(mine);
  each = __builtin_amdgcn_readfirstlane(each);
  int turn = 0;        // tiles that a wavefront has alone
  // Tiles of this slot that the piece has passed, and those that it holds in whole
  // groups of one for each wavefront.
  int k = 0, groups = 0;
  auto count_groups = [&]() __attribute__((always_inline)) {
    const int first = at < 0 ? 1 : 0;   // (begun before the piece)
    const int here = per_slot - (head * sides.turns + round);
    const int whole = ratio(mine - at, kOverhead + steps);
    k = -first;
    groups = ((here < whole ? here : whole) - first) / kAttnWaves * kAttnWaves;
  };
  count_groups();
  // a workgroup has two parts at most: of a tile that began before its piece of the
  // line, and of one that goes on behind it
  const uint32_t size = part_bytes(a.group, kDims);
  auto part_at = [&](int of, bool goes_on) __attribute__((always_inline)) {
    return (2u * static_cast<uint32_t>(of * sides.side + beside) + (goes_on ? 1u : 0u)) * size;
  };
  const __amdgpu_buffer_rsrc_t rs = row_buffer(parts, parts_bytes);
  while (at < mine) {
    const int query0 = (round * sides.side + beside) * 16;
    const int queries = a.group - query0 < 16 ? a.group - query0 : 16;   // (none: zero or less)
    const int row0 = slot * a.q_heads + head * a.group + query0;
    // this workgroup's steps of the tile
    const int step0 = at + kOverhead;
    const int lo = cut(-step0, steps);
    const int hi = cut(mine - step0, steps);
    if (steps == 0 && at >= 0) {   // (no turn of a loop where there are no queries)
      for (int i = tid; i < queries * a.c.head_dim / 4; i += NT)
        store4<T>(a.out, static_cast<int64_t>(row0) * a.c.head_dim + i * 4, floatx4{0.f, 0.f, 0.f, 0.f});
      if (a.lse != nullptr && tid < queries) a.lse[row0 + tid] = -__builtin_inff();
    }
    // Short tiles cost little but the wait for their data: each wavefront takes tiles
    // of its own, without barriers and LDS; longer ones only where the piece holds one
    // for every wavefront, of one length (200 slots of 350 tokens, 16 heads of 16 bf16:
    // 55 us, 63 without; 128 of 400, 32 heads of 72: 122 and 120).
    bool alone = lo == 0 && hi == steps;
    if (steps <= kFew) alone = alone && (steps == 1 || 2 * (kOverhead + steps) <= each);
    else alone = alone && k >= 0 && k < groups;
    ++k;
    if (lo < hi && queries > 0 && !(alone && turn++ % kAttnWaves != wv)) {
      W w;
      w.clear();
      load_queries(a, w, slot, head, query0);
      walk(a, w, slot, head, seen, known, alone ? 0 : lo + wv, hi, alone ? 1 : kAttnWaves, bad);
      const float l = sum_of_groups(w.l);
      if (alone) {
        if (c < queries) {
          const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
          for (int t = 0; t < W::OT; ++t) {
            const int d = 16 * t + 4 * g;
            const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
            if (d < a.c.head_dim)
              store4<T>(a.out, static_cast<int64_t>(row0 + c) * a.c.head_dim + d, l == 0.0f ? zero : w.o[t] * inv);
          }
          if (g == 0 && a.lse != nullptr)
            a.lse[row0 + c] = l == 0.0f ? -__builtin_inff() : (w.m + __builtin_amdgcn_logf(l)) * kLn2;
        }
      } else {
        __syncthreads();   // the tile before this one has left LDS
        if (g == 0) {
          sh.m[wv][c] = w.m;
          sh.l[wv][c] = l;
        }
#pragma unroll
        for (int t = 0; t < W::OT; ++t) *reinterpret_cast<floatx4*>(&sh.o[wv][c][16 * t + 4 * g]) = w.o[t];
        __syncthreads();
        bool ends = lo == 0 && hi == steps;
        if (!ends) {
          store_part(sh, queries, rs, part_at(piece, lo == 0));
          // the workgroups that have the tile's first part and its last
          const int w0 = piece + ratio(step0 + kPart - 1, each);
          const int w1 = piece + ratio(step0 + steps - kPart, each);
          uint32_t* ticket = tickets + (w1 * sides.side + beside);
          wait_vmcnt<0>();
          __syncthreads();
          if (tid == 0)
            is_last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                      static_cast<uint32_t>(w1 - w0);
          __syncthreads();
          ends = is_last != 0;
          if (ends) {
            const int n = w1 - w0 + 1;
            auto part = [&](int p) __attribute__((always_inline)) { return part_at(w0 + p, p == 0); };
            if (n <= kFewParts) collect<kFewParts / kAttnWaves>(sh, weights, queries, n, rs, part);
            else collect<kTurn / kAttnWaves>(sh, weights, queries, n, rs, part);
            if (tid == 0) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          }
        }
        if (ends) finish<T>(a, sh, row0, queries);
      }
    }
    at += kOverhead + steps;
    if (++round == sides.turns) {
      round = 0;
      if (++head == a.c.heads) {
        head = 0;
        if (at >= mine) break;
        ++slot;
        seen = seen_of(a, slot);
        known.begin(a, slot, seen);
        steps = __builtin_amdgcn_readfirstlane(steps_of(seen));
        count_groups();
      }
    }
  }
  if (bad != 0 && a.flags != nullptr) atomicOr(a.flags, bad);
}

uint32_t parts_bytes(int32_t group, int dims) { return 2u * kWorkers * part_bytes(group, dims); }

template <typename T, int NP, bool ALONE>
hipError_t launch(const AttnArgs& a, void* workspace, hipStream_t st) {
  const Sides sides = sides_of(a.group);
  // no more workgroups than the longest line would have pieces
  constexpr int SB = Wave<T, NP, ALONE>::SB;
  const int64_t longest = kOverhead + 1 + (static_cast<int64_t>(a.c.max_pages) * a.c.page / kBlockTokens + SB) / SB;
  const int64_t pieces = (longest * a.c.n_slots * a.c.heads * sides.turns + kLeast - 1) / kLeast;
  const int64_t taken = pieces < sides.pieces ? (pieces + kXcds - 1) / kXcds * kXcds : sides.pieces;
  uint32_t* tickets = static_cast<uint32_t*>(workspace);
  k_attn<T, NP, ALONE><<<static_cast<unsigned>(taken * sides.side), kAttnWaves * kWave, 0, st>>>(
      a, sides, tickets, static_cast<char*>(workspace) + FM_ATTN_TICKET_BYTES,
      parts_bytes(a.group, NP * kRowPiece / static_cast<int>(sizeof(T))));
  return hipGetLastError();
}

template <typename T, int NP = 1>
hipError_t launch_pieces(const AttnArgs& a, void* workspace, hipStream_t st) {
  if constexpr (NP > kMaxHeadDim * static_cast<int>(sizeof(T)) / kRowPiece)
    return hipErrorInvalidValue;
  else if (a.c.pieces != NP)
    return launch_pieces<T, NP + 1>(a, workspace, st);
  else
    return a.group <= 16 ? launch<T, NP, true>(a, workspace, st) : launch<T, NP, false>(a, workspace, st);
}

}  // namespace

static_assert(kWorkers * sizeof(uint32_t) <= FM_ATTN_TICKET_BYTES && FM_ATTN_TICKET_BYTES % kAlign == 0, "tickets");

bool attn_fits(const fm_kv_cache& c, int32_t q_heads) {
  // a workgroup's places on the line are int32, of a step per block at most
  const int64_t tile = kOverhead + 1 + static_cast<int64_t>(c.max_pages) * c.page / kBlockTokens;
  const Sides sides = sides_of(q_heads / c.heads);
  const int64_t tiles = static_cast<int64_t>(c.n_slots) * c.heads * sides.turns;
  return tiles <= (static_cast<int64_t>(sides.pieces) << 28) / tile;
}

size_t attn_workspace_bytes(const fm_kv_cache& c, int32_t q_heads) {
  const int dims = kv_pieces(c.head_dim, c.dtype) * kRowPiece / (c.dtype == FM_BF16 ? 2 : 4);
  return FM_ATTN_TICKET_BYTES + align_up(parts_bytes(q_heads / c.heads, dims), kAlign);
}

hipError_t launch_attn(const AttnArgs& a, fm_dtype dt, void* workspace, hipStream_t st) {
  return dt == FM_BF16 ? launch_pieces<uint16_t>(a, workspace, st) : launch_pieces<float>(a, workspace, st);
}

}  // namespace fm
