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

// The wavefronts' maxima, sums and outputs of a tile, through LDS.
template <int NP4>   // dimensions of a padded row
struct Joined {
  static constexpr int kLd = NP4 + 4;
  float m[kAttnWaves][16], l[kAttnWaves][16];
  float o[kAttnWaves][16][kLd];
};

// A workgroup per slot, key head and tile of 16 of its queries.
template <typename T, int NP>
__global__ void __launch_bounds__(kAttnWaves* kWave) k_attn(AttnArgs a) {
  using W = Wave<T, NP>;
  constexpr int kDims = NP * kRowPiece / static_cast<int>(sizeof(T));
  __shared__ Joined<kDims> sh;
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int c = lane % 16, g = lane / 16;
  const int tile = static_cast<int>(blockIdx.x) % a.tiles;
  const int head = static_cast<int>(blockIdx.x) / a.tiles % a.c.heads;
  const int slot = static_cast<int>(blockIdx.x) / a.tiles / a.c.heads;
  const Seen seen = seen_of(a, slot);
  const int queries = a.group - tile * 16 < 16 ? a.group - tile * 16 : 16;
  const int q0 = head * a.group + tile * 16;
  uint32_t bad = 0;

  W w;
  w.clear();
  if (!seen.none()) {
    load_queries<T, NP>(a, w, slot, head, tile);
    const int blocks = (seen.hi + kBlockTokens - 1) / kBlockTokens - seen.lo / kBlockTokens;
    walk<T, NP>(a, w, slot, head, seen, wv, (blocks + W::SB - 1) / W::SB, kAttnWaves, bad);
  }
  const float l = sum_of_groups(w.l);
  if (g == 0) {
    sh.m[wv][c] = w.m;
    sh.l[wv][c] = l;
  }
#pragma unroll
  for (int t = 0; t < W::OT; ++t) *reinterpret_cast<floatx4*>(&sh.o[wv][c][16 * t + 4 * g]) = w.o[t];
  __syncthreads();
  const int quads = a.c.head_dim / 4;
  for (int i = tid; i < queries * quads; i += kAttnWaves * kWave) {
    const int qi = i / quads, d = i % quads * 4;
    float top = -__builtin_inff();
#pragma unroll
    for (int u = 0; u < kAttnWaves; ++u) top = fmaxf(top, sh.m[u][qi]);
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    float all = 0.0f;
#pragma unroll
    for (int u = 0; u < kAttnWaves; ++u) {
      const float mu = sh.m[u][qi];
      // (a wavefront that saw no score has the maximum minus infinity)
      const float f = mu == -__builtin_inff() ? (sh.l[u][qi] == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f(mu - top);
      all += f * sh.l[u][qi];
      sum += f * *reinterpret_cast<const floatx4*>(&sh.o[u][qi][d]);
    }
    const int64_t at = (static_cast<int64_t>(slot) * a.q_heads + q0 + qi);
    const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
    store4<T>(a.out, at * a.c.head_dim + d, all == 0.0f ? zero : sum / all);
    if (d == 0 && a.lse != nullptr)
      a.lse[at] = all == 0.0f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(all)) * kLn2;
  }
  if (bad != 0 && a.flags != nullptr) atomicOr(a.flags, bad);
}

template <typename T, int NP>
hipError_t launch(const AttnArgs& a, hipStream_t st) {
  k_attn<T, NP><<<static_cast<unsigned>(a.c.heads * a.tiles * a.c.n_slots), kAttnWaves * kWave, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t attn_workspace_bytes(const fm_kv_cache& c, int32_t q_heads) { return kAlign; }

hipError_t launch_attn(const AttnArgs& a, fm_dtype dt, void* workspace, hipStream_t st) {
  if (dt == FM_BF16) {
    switch (a.c.pieces) {
      case 1: return launch<uint16_t, 1>(a, st);
      case 2: return launch<uint16_t, 2>(a, st);
      case 3: return launch<uint16_t, 3>(a, st);
      case 4: return launch<uint16_t, 4>(a, st);
      case 5: return launch<uint16_t, 5>(a, st);
      case 6: return launch<uint16_t, 6>(a, st);
      case 7: return launch<uint16_t, 7>(a, st);
      case 8: return launch<uint16_t, 8>(a, st);
      default: return hipErrorInvalidValue;
    }
  }
  switch (a.c.pieces) {
    case 1: return launch<float, 1>(a, st);
    case 2: return launch<float, 2>(a, st);
    case 3: return launch<float, 3>(a, st);
    case 4: return launch<float, 4>(a, st);
    case 5: return launch<float, 5>(a, st);
    case 6: return launch<float, 6>(a, st);
    case 7: return launch<float, 7>(a, st);
    case 8: return launch<float, 8>(a, st);
    case 9: return launch<float, 9>(a, st);
    case 10: return launch<float, 10>(a, st);
    case 11: return launch<float, 11>(a, st);
    case 12: return launch<float, 12>(a, st);
    case 13: return launch<float, 13>(a, st);
    case 14: return launch<float, 14>(a, st);
    case 15: return launch<float, 15>(a, st);
    case 16: return launch<float, 16>(a, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace fm
