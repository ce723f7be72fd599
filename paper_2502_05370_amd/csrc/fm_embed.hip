// Token embeddings: the rows of a batch of tokens, each request's mean row (the
// semantic query of Section 4.2.1), and the table's gradient.
//
// All three move rows and add a few of them, one or two operations per element:
// memory bounds them.  Rows are read 16 bytes per lane, whatever their
// alignment (gfx950 takes a vector access at any element's address), so that odd
// widths run on the same path; the elements past the last whole vector of a row
// go one by one.
#include "fm_device.h"
#include "fm_internal.h"

namespace fm {

namespace {

// N elements of a row, aligned to one element only; by default 16 bytes.
template <typename T, int n = 16 / sizeof(T)>
struct Vec {
  static constexpr int N = n;
  typedef T raw __attribute__((ext_vector_type(n)));
  typedef raw mem __attribute__((aligned(sizeof(T))));
};

__device__ __forceinline__ float widen(uint16_t h) { return bf16_to_f32(h); }
__device__ __forceinline__ float widen(float f) { return f; }
template <typename T>
__device__ __forceinline__ T narrow(float f) {
  if constexpr (sizeof(T) == 2) return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f));   // to nearest even
  else return f;
}

// The n <= N elements of a row at p (n < N only at the end of a row), zeros past
// them.
template <typename T, int N = Vec<T>::N>
__device__ __forceinline__ typename Vec<T, N>::raw load_part(const T* p, int n) {
  typename Vec<T, N>::raw v = {};
  if (n >= N) {
    v = *reinterpret_cast<const typename Vec<T, N>::mem*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (i < n) v[i] = p[i];
  }
  return v;
}
// STREAM: the row is not read again soon (a hint to the caches).
template <bool STREAM, typename T, int N = Vec<T>::N>
__device__ __forceinline__ void store_part(T* p, typename Vec<T, N>::raw v, int n) {
  if (n >= N) {
    typename Vec<T, N>::mem* q = reinterpret_cast<typename Vec<T, N>::mem*>(p);
    if constexpr (STREAM) __builtin_nontemporal_store(v, q);
    else *q = v;
  } else {
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (i < n) p[i] = v[i];
  }
}

// The row that a token selects, or -1 (padding, or past the table: flagged).
__device__ __forceinline__ int row_of(int32_t tok, int32_t V, uint32_t* flags) {
  if (tok < V) return tok < 0 ? -1 : tok;
  if (flags != nullptr) atomicOr(flags, static_cast<uint32_t>(FM_FLAG_INDEX_RANGE));
  return -1;
}

// ---------------------------------------------------------------- lookup

constexpr int kLookThreads = 256;

// A group of `lanes` lanes copies U vectors per lane of one token's row, so a
// row spans gridDim.y groups.  65,536 rows of 4,096 bf16 (709 MB with each distinct
// row read once): 140 us, the rate of a large copy (4.96 TB/s); with plain stores
// 150.
template <typename T, int U>
__global__ void __launch_bounds__(kLookThreads) k_embed_lookup(const T* __restrict__ table, int32_t V, int32_t d,
                                                               const int32_t* __restrict__ tokens, int32_t n_tok,
                                                               float scale, T* __restrict__ out, int lanes_log,
                                                               uint32_t* __restrict__ flags) {
  constexpr int N = Vec<T>::N;
  const int lanes = 1 << lanes_log;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kLookThreads >> lanes_log) + (threadIdx.x >> lanes_log);
  if (t >= n_tok) return;
  const int row = row_of(tokens[t], V, flags);
  if (row < 0) scale = 0.0f;   // zeros whatever the scale
  const int col0 = (static_cast<int>(blockIdx.y) * U * lanes + (threadIdx.x & (lanes - 1))) * N;
  const T* src = table + static_cast<int64_t>(row < 0 ? 0 : row) * d;
  T* dst = out + t * d;
  typename Vec<T>::raw v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = col0 + u * lanes * N;
    v[u] = load_part(src + c, row < 0 ? 0 : d - c);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = col0 + u * lanes * N;
    if (c >= d) break;
#pragma unroll
    for (int i = 0; i < N; ++i) v[u][i] = narrow<T>(widen(v[u][i]) * scale);
    store_part<true>(dst + c, v[u], d - c);
  }
}

template <typename T>
void lookup(const void* table, int32_t V, int32_t d, const int32_t* tokens, int32_t n_tok, float scale, void* out,
            uint32_t* flags, hipStream_t st) {
  const int nv = (d + Vec<T>::N - 1) / Vec<T>::N;
  int lg = 0;
  while (lg < 6 && (1 << lg) < nv) ++lg;
  const int groups = kLookThreads >> lg;
  const unsigned gx = static_cast<unsigned>((static_cast<int64_t>(n_tok) + groups - 1) / groups);
  const unsigned gy = static_cast<unsigned>((nv + 4 * (1 << lg) - 1) / (4 * (1 << lg)));
  k_embed_lookup<T, 4><<<dim3(gx, gy), kLookThreads, 0, st>>>(static_cast<const T*>(table), V, d, tokens, n_tok, scale,
                                                              static_cast<T*>(out), lg, flags);
}

// ---------------------------------------------------------------- pool

constexpr int kPoolTokens = 1024;   // tokens of a request staged at a time

// One workgroup of NW wavefronts per (request, block of columns): CL lanes
// hold the block's columns, the wavefronts' 64 / CL lane groups take the
// request's tokens in turn, and their sums are joined in a fixed order.  The
// column block is the fastest grid index: where the blocks are a multiple of 8,
// each XCD's L2 sees one eighth of the columns of the frequent rows.  1,024 requests
// of 300 tokens on average, 2,048 columns: 100 us for 1.26 GB of rows, of which
// text frequencies leave about 0.45 GB to the memory behind the L2; vectors of 8
// bytes, scalar row addresses and other block widths stay within 97-146 us.
template <typename T, int CL, int NW>
__global__ void __launch_bounds__(NW * kWave) k_embed_pool(const T* __restrict__ table, int32_t V, int32_t d,
                                                           const int32_t* __restrict__ tokens, int32_t n_tok,
                                                           const int32_t* __restrict__ offsets, int n_blk, float scale,
                                                           uint16_t* __restrict__ out, uint32_t* __restrict__ flags) {
  constexpr int N = Vec<T>::N;
  constexpr int G = kWave / CL;    // token groups of a wavefront
  constexpr int U = 8;             // rows in flight per lane
  __shared__ int32_t rows[kPoolTokens];
  __shared__ float part[NW][CL * N + 4];
  __shared__ int32_t n_live;
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int wv = tid / kWave;
  const int b = blockIdx.x / n_blk;
  const int col = (static_cast<int>(blockIdx.x % n_blk) * CL + lane % CL) * N;
  const int have = d - col;         // elements of the row from this lane's columns on
  auto clamp = [&](int o) { return o < 0 ? 0 : (o > n_tok ? n_tok : o); };
  const int t0 = clamp(offsets[b]);
  const int t1 = clamp(offsets[b + 1]);
  if (tid == 0) n_live = 0;
  float acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = 0.0f;
  int live = 0;
  for (int c0 = t0; c0 < t1; c0 += kPoolTokens) {
    const int n = t1 - c0 < kPoolTokens ? t1 - c0 : kPoolTokens;
    __syncthreads();
    for (int i = tid; i < n; i += NW * kWave) {
      const int r = row_of(tokens[c0 + i], V, flags);
      rows[i] = r;
      live += r >= 0 ? 1 : 0;
    }
    __syncthreads();
    for (int i0 = wv * G + lane / CL; i0 < n; i0 += U * NW * G) {
      typename Vec<T>::raw v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * NW * G;
        const int r = i < n ? rows[i] : -1;
        v[u] = load_part(table + static_cast<int64_t>(r < 0 ? 0 : r) * d + col, r < 0 ? 0 : have);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] += widen(v[u][i]);
    }
  }
  // (every lane holds a part of the count; the column blocks count alike)
#pragma unroll
  for (int m = kWave / 2; m >= 1; m >>= 1) live += __shfl_xor(live, m, kWave);
  if (t1 <= t0) __syncthreads();   // n_live is cleared
  if (lane == 0 && live != 0) atomicAdd(&n_live, live);
#pragma unroll
  for (int m = CL; m < kWave; m <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] += __shfl_xor(acc[i], m, kWave);
  if (lane < CL)
#pragma unroll
    for (int i = 0; i < N; ++i) part[wv][lane * N + i] = acc[i];
  __syncthreads();
  if (tid >= CL || have <= 0) return;
  const float w = n_live > 0 ? scale / static_cast<float>(n_live) : 0.0f;
  uint16_t* dst = out + static_cast<int64_t>(b) * d + col;
  uint16_t r[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float s = 0.0f;
#pragma unroll
    for (int u = 0; u < NW; ++u) s += part[u][tid * N + i];
    r[i] = n_live > 0 ? narrow<uint16_t>(s * w) : static_cast<uint16_t>(0);
  }
  if constexpr (N == 8) {
    Vec<uint16_t>::raw v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = r[i];
    store_part<false>(dst, v, have);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < have) dst[i] = r[i];
  }
}

template <typename T, int CL>
void pool_cl(const void* table, int32_t V, int32_t d, const int32_t* tokens, int32_t T_, const int32_t* offsets,
             int32_t B, float scale, uint16_t* out, uint32_t* flags, int n_blk, hipStream_t st) {
  const unsigned grid = static_cast<unsigned>(static_cast<int64_t>(B) * n_blk);
  k_embed_pool<T, CL, 4><<<grid, 4 * kWave, 0, st>>>(static_cast<const T*>(table), V, d, tokens, T_, offsets, n_blk,
                                                     scale, out, flags);
}

template <typename T>
void pool(const void* table, int32_t V, int32_t d, const int32_t* tokens, int32_t T_, const int32_t* offsets, int32_t B,
          float scale, uint16_t* out, uint32_t* flags, hipStream_t st) {
  // Blocks of 32 lanes' columns, or of 8 where those would be fewer than 1,024
  // workgroups (four per CU): four times the workgroups, with a quarter of the
  // rows each lane group adds one after the other.  That helps requests of many
  // tokens (us, 32 and 8 lanes: 8 requests of 300 tokens of 2,048 bf16 7.8 and 5.8,
  // of 4,096 7.8 and 6.3) up to some 256 workgroups of 32 lanes (32 requests of
  // 2,048 8.8 and 8.1, 64 11.2 and 13.4, 128 16.8 and 20.7), and costs short ones (8
  // requests of 37 tokens of 4,096 4.0 and 5.1).
  const int nv = (d + Vec<T>::N - 1) / Vec<T>::N;
  auto blocks = [&](int cl) { return (nv + cl - 1) / cl; };
  if (static_cast<int64_t>(B) * blocks(32) >= 1024)
    pool_cl<T, 32>(table, V, d, tokens, T_, offsets, B, scale, out, flags, blocks(32), st);
  else
    pool_cl<T, 8>(table, V, d, tokens, T_, offsets, B, scale, out, flags, blocks(8), st);
}

// ---------------------------------------------------------------- gradient

// Three launches: the rows' lists are cleared, the batch's tokens are listed by
// row, and the rows are written; two where one workgroup lists the whole batch,
// whose table of distinct tokens then stands in for the rows' lists.  A frequent token's row (more than kFrequent
// tokens select it) is summed by whole workgroups, every other row by one
// wavefront.
constexpr int kFrequent = 32;
constexpr int kListTokens = 1024;   // tokens that a workgroup lists
constexpr int kListSlots = 2048;    // slots of its table of distinct tokens
constexpr int kRowThreads = 256;
constexpr int kWaveRows = 4;        // rows of one wavefront
constexpr int kFreqLanes = 32;      // lanes over the columns of a frequent row's block
constexpr int kFreqGroups = 512;    // workgroups that share the frequent rows
constexpr int kFreqList = 256;      // positions from which a wavefront adds the rows it has listed
constexpr int kFreqSpace = kFreqList + 1024;

// What the batch holds of a row: the last token listed (-1: none) and how many.
struct RowList {
  int32_t head, count;
};

// A slot of the table of distinct tokens.
struct Distinct {
  int32_t row;       // -1: free
  RowList list;
};
__device__ __forceinline__ uint32_t first_slot(int32_t row) {
  static_assert(kListSlots == 1 << 11, "the product's upper 11 bits");
  return static_cast<uint32_t>(row) * 2654435761u >> 21;
}

struct GradScratch {
  RowList* rows;     // [V], or [kListSlots] Distinct
  int32_t* next;     // [T] the token listed before it in its row
  int32_t* freq;     // [T / kFrequent] the frequent rows
  int32_t* n_freq;
};

size_t scratch_parts(int32_t T, int32_t V, GradScratch* s, char* base) {
  const size_t rows = align_up(sizeof(int32_t), kAlign);
  const size_t next = rows + align_up(static_cast<size_t>(V) * sizeof(RowList), kAlign);
  const size_t freq = next + align_up(static_cast<size_t>(T) * sizeof(int32_t), kAlign);
  if (s != nullptr) {
    s->n_freq = reinterpret_cast<int32_t*>(base);
    s->rows = reinterpret_cast<RowList*>(base + rows);
    s->next = reinterpret_cast<int32_t*>(base + next);
    s->freq = reinterpret_cast<int32_t*>(base + freq);
  }
  return freq + align_up((static_cast<size_t>(T) / kFrequent + 1) * sizeof(int32_t), kAlign);
}

__global__ void __launch_bounds__(256) k_grad_clear(GradScratch s, int32_t V) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i == 0) *s.n_freq = 0;
  if (i < V) s.rows[i] = RowList{-1, 0};
}

// Each row's tokens become a list in an order that depends on timing; the sums
// below put the positions back in order.  A workgroup first lists its own tokens
// in a table in LDS and then joins each distinct token's list to the row's: an
// atomic per occurrence costs 18 ns on the rows of frequent tokens (65,536
// tokens of text frequencies: 40.6 us for this launch).
template <bool WHOLE>   // one workgroup lists the whole batch
__global__ void __launch_bounds__(kListTokens) k_grad_list(GradScratch s, const int32_t* __restrict__ tokens,
                                                           int32_t n_tok, int32_t V, uint32_t* __restrict__ flags) {
  __shared__ int32_t key[kListSlots], head[kListSlots], tail[kListSlots], count[kListSlots], n_freq;
  const int tid = threadIdx.x;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kListTokens + tid;
  const int row = t < n_tok ? row_of(tokens[t], V, flags) : -1;
  for (int i = tid; i < kListSlots; i += kListTokens) {
    key[i] = head[i] = -1;
    count[i] = 0;
  }
  if (tid == 0) n_freq = 0;
  __syncthreads();
  if (row >= 0) {
    // at most kListTokens of the slots are taken, so that a free one is met
    uint32_t i = first_slot(row);
    for (;;) {
      const int32_t k = atomicCAS(&key[i], -1, row);
      if (k == -1 || k == row) break;
      i = (i + 1) % kListSlots;
    }
    const int32_t before = atomicExch(&head[i], static_cast<int32_t>(t));
    if (before < 0) tail[i] = static_cast<int32_t>(t);
    else s.next[t] = before;
    atomicAdd(&count[i], 1);
  }
  __syncthreads();
  for (int i = tid; i < kListSlots; i += kListTokens) {
    const int32_t r = key[i];
    if constexpr (WHOLE) {
      reinterpret_cast<Distinct*>(s.rows)[i] = Distinct{r, {head[i], count[i]}};
      if (r >= 0 && count[i] > kFrequent) s.freq[atomicAdd(&n_freq, 1)] = r;
      continue;
    }
    if (r < 0) continue;
    s.next[tail[i]] = atomicExch(&s.rows[r].head, head[i]);
    const int32_t n = atomicAdd(&s.rows[r].count, count[i]);
    if (n <= kFrequent && n + count[i] > kFrequent) s.freq[atomicAdd(s.n_freq, 1)] = r;
  }
  if constexpr (WHOLE) {
    __syncthreads();
    if (tid == 0) *s.n_freq = n_freq;
  }
}

// What the batch holds of a row.
__device__ __forceinline__ RowList row_list(const GradScratch& s, int64_t row, bool table) {
  if (!table) return s.rows[row];
  const Distinct* t = reinterpret_cast<const Distinct*>(s.rows);
  for (uint32_t i = first_slot(static_cast<int32_t>(row));; i = (i + 1) % kListSlots) {
    const Distinct d = t[i];   // (at most half of the slots are taken: a free one is met)
    if (d.row == static_cast<int32_t>(row)) return d.list;
    if (d.row < 0) return RowList{-1, 0};
  }
}

// N sums into a row of the gradient.
template <typename G, int N>
__device__ __forceinline__ void put_row(G* dst, const float* acc, int n, float scale, bool accumulate, bool any) {
  typename Vec<G, N>::raw v = {};
  if (accumulate) v = load_part<G, N>(dst, n);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float s = any ? acc[i] * scale : 0.0f;
    v[i] = narrow<G>(accumulate ? widen(v[i]) + s : s);
  }
  store_part<true, G, N>(dst, v, n);
}

struct GradArgs {
  GradScratch s;
  const int32_t* tokens;
  int32_t n_tok, V, d;
  float scale;
  bool accumulate;
  bool table;        // the lists stand in the table of one workgroup's distinct tokens
  int freq_groups;   // workgroups of the frequent rows, before those of the others
};

// Vectors of a row: 16 bytes of the wider type.
template <typename T, typename G>
constexpr int vec_elems() {
  return 16 / (sizeof(T) > sizeof(G) ? sizeof(T) : sizeof(G));
}

// kWaveRows rows of at most kFrequent tokens by one wavefront.  The lanes read
// the rows' positions off their lists side by side and put them in order by
// rank; then the rows of dout are added in that order, the first of the next row
// on its way while this one is written.  A row without a token is written as
// zeros, or left alone when accumulating.
template <typename T, typename G>
__device__ __forceinline__ void rare_rows(const GradArgs& a, const T* __restrict__ dout, int64_t row0,
                                          G* __restrict__ dtable, int32_t (*ord)[kFrequent], int32_t* unordered) {
  constexpr int N = vec_elems<T, G>();
  constexpr int U = 4;
  constexpr int kSpan = U * kWave * N;   // columns of one pass
  const int lane = threadIdx.x % kWave;
  RowList mine = {-1, 0};
  if (lane < kWaveRows && row0 + lane < a.V) mine = row_list(a.s, row0 + lane, a.table);
  if (mine.count > kFrequent) mine.count = -1;
  const int longest = [&] {
    int m = 0;
#pragma unroll
    for (int j = 0; j < kWaveRows; ++j) {
      const int n = __builtin_amdgcn_readlane(mine.count, j);
      m = n > m ? n : m;
    }
    return m;
  }();
  {
    int p = mine.head;
    for (int i = 0; i < longest; ++i) {
      if (i < mine.count) {
        unordered[lane * kFrequent + i] = p;
        if (i + 1 < mine.count) p = a.s.next[p];
      }
    }
    wait_lgkm0();
  }
#pragma unroll
  for (int j = 0; j < kWaveRows; ++j) {
    const int n = __builtin_amdgcn_readlane(mine.count, j);
    if (n < 1) continue;
    const int pos = lane < n ? unordered[j * kFrequent + lane] : 0;
    int rank = 0;
    for (int i = 0; i < n; ++i) rank += __builtin_amdgcn_readlane(pos, i) < pos ? 1 : 0;
    if (lane < n) ord[j][rank] = pos;
  }
  wait_lgkm0();
  const int passes = (a.d + kSpan - 1) / kSpan;
  auto fetch = [&](typename Vec<T, N>::raw (&v)[U], int j, int i, int pass) __attribute__((always_inline)) {
    const T* src = dout + static_cast<int64_t>(ord[j][i]) * a.d;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = pass * kSpan + (u * kWave + lane) * N;
      v[u] = load_part<T, N>(src + c, a.d - c);
    }
  };
  // rows with tokens first, so that their loads start at once
  for (int pass = 0; pass < passes; ++pass) {
    typename Vec<T, N>::raw ahead[U];
    int j = 0;
    int n = 0;
    auto next_row = [&](int from) __attribute__((always_inline)) {
      for (int q = from; q < kWaveRows; ++q)
        if (__builtin_amdgcn_readlane(mine.count, q) > 0) return q;
      return kWaveRows;
    };
    j = next_row(0);
    if (j < kWaveRows) fetch(ahead, j, 0, pass);
    while (j < kWaveRows) {
      n = __builtin_amdgcn_readlane(mine.count, j);
      float acc[U][N];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < N; ++i) acc[u][i] = widen(ahead[u][i]);
      for (int i = 1; i < n; ++i) {
        typename Vec<T, N>::raw v[U];
        fetch(v, j, i, pass);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < N; ++e) acc[u][e] += widen(v[u][e]);
      }
      const int after = next_row(j + 1);
      if (after < kWaveRows) fetch(ahead, after, 0, pass);
      G* dst = dtable + (row0 + j) * a.d;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = pass * kSpan + (u * kWave + lane) * N;
        if (c < a.d) put_row<G, N>(dst + c, acc[u], a.d - c, a.scale, a.accumulate, true);
      }
      j = after;
    }
    if (a.accumulate) continue;
    for (int q = 0; q < kWaveRows && row0 + q < a.V; ++q) {
      if (__builtin_amdgcn_readlane(mine.count, q) != 0) continue;
      G* dst = dtable + (row0 + q) * a.d;
      const float none[N] = {};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = pass * kSpan + (u * kWave + lane) * N;
        if (c < a.d) put_row<G, N>(dst + c, none, a.d - c, a.scale, false, false);
      }
    }
  }
}

// Frequent rows: a workgroup takes (row, block of columns) units in turn.  Every
// unit reads the whole batch's tokens, so that their cost grows with the batch's
// length times the number of frequent rows: with text frequencies over 128,000
// rows of 2,048 bf16 0.21 ms for 65,536 tokens (178 frequent rows), 1.06 for 262,144
// (754) and 13.2 for 1,048,576 (2,977), which move 0.8, 1.6 and 4.8 GB.  Its
// wavefronts share the batch in equal ranges, list their tokens of the row in an
// order that the tokens alone decide, and the lane groups add the listed rows in
// turn; the groups' and wavefronts' sums are joined in a fixed order.
template <typename T, typename G>
__device__ __forceinline__ void frequent_rows(const GradArgs& a, const T* __restrict__ dout, G* __restrict__ dtable,
                                              int32_t (*list)[kFreqSpace], float* part) {
  constexpr int N = vec_elems<T, G>();
  constexpr int NW = kRowThreads / kWave;
  constexpr int GR = kWave / kFreqLanes;
  constexpr int U = 8;      // rows in flight per lane
  constexpr int TB = 4;     // loads of four tokens in flight
  constexpr int kLd = kFreqLanes * N + 4;
  typedef int32_t int4v __attribute__((ext_vector_type(4)));
  typedef int4v int4m __attribute__((aligned(4)));
  static_assert(kFreqSpace >= kFreqList + TB * 4 * kWave, "a batch of loads fits the list");
  const int lane = threadIdx.x % kWave;
  const int wv = threadIdx.x / kWave;
  const int n_blk = (a.d + kFreqLanes * N - 1) / (kFreqLanes * N);
  const int64_t units = static_cast<int64_t>(*a.s.n_freq) * n_blk;
  const int share = (a.n_tok + NW * 4 - 1) / (NW * 4) * 4;   // tokens per wavefront
  const int first = wv * share;
  const int last = first + share < a.n_tok ? first + share : a.n_tok;
  for (int64_t u0 = blockIdx.x; u0 < units; u0 += a.freq_groups) {
    const int32_t row = a.s.freq[u0 / n_blk];
    const int col = (static_cast<int>(u0 % n_blk) * kFreqLanes + lane % kFreqLanes) * N;
    const int have = a.d - col;
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.0f;
    int n = 0;   // listed positions
#pragma unroll 1
    for (int t0 = first; t0 < last; t0 += TB * 4 * kWave) {
      int4v tok[TB];
#pragma unroll
      for (int b = 0; b < TB; ++b) {
        const int t = t0 + (b * kWave + lane) * 4;
        if (t + 3 < last) {
          tok[b] = *reinterpret_cast<const int4m*>(a.tokens + t);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) tok[b][i] = t + i < last ? a.tokens[t + i] : -1;
        }
      }
#pragma unroll
      for (int b = 0; b < TB; ++b) {
        uint64_t m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = __ballot(tok[b][i] == row);
        if ((m[0] | m[1] | m[2] | m[3]) == 0) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if ((m[i] >> lane) & 1ull)
            list[wv][n + __popcll(m[i] & ((1ull << lane) - 1ull))] = t0 + (b * kWave + lane) * 4 + i;
          n += __popcll(m[i]);
        }
      }
      if (n < kFreqList && t0 + TB * 4 * kWave < last) continue;
      wait_lgkm0();
#pragma unroll 1
      for (int i0 = lane / kFreqLanes; i0 < n; i0 += U * GR) {
        typename Vec<T, N>::raw v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + u * GR;
          v[u] = load_part<T, N>(dout + static_cast<int64_t>(i < n ? list[wv][i] : 0) * a.d + col, i < n ? have : 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < N; ++i) acc[i] += widen(v[u][i]);
      }
      n = 0;
    }
#pragma unroll
    for (int m = kFreqLanes; m < kWave; m <<= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] += __shfl_xor(acc[i], m, kWave);
    if (lane < kFreqLanes)
#pragma unroll
      for (int i = 0; i < N; ++i) part[wv * kLd + lane * N + i] = acc[i];
    __syncthreads();
    if (wv == 0 && lane < kFreqLanes && have > 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        acc[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) acc[i] += part[w * kLd + lane * N + i];
      }
      put_row<G, N>(dtable + static_cast<int64_t>(row) * a.d + col, acc, have, a.scale, a.accumulate, true);
    }
    __syncthreads();
  }
}

// The frequent rows' workgroups come first in the grid, so that their longer
// work overlaps the other rows', which memory bounds.
template <typename T, typename G>
__global__ void __launch_bounds__(kRowThreads, 5) k_grad_rows(GradArgs a, const T* __restrict__ dout,
                                                              G* __restrict__ dtable) {
  constexpr int NW = kRowThreads / kWave;
  __shared__ int32_t list[NW][kFreqSpace];
  __shared__ float part[NW * (kFreqLanes * vec_elems<T, G>() + 4)];
  if (static_cast<int>(blockIdx.x) < a.freq_groups) {
    frequent_rows<T, G>(a, dout, dtable, list, part);
    return;
  }
  const int wv = threadIdx.x / kWave;
  static_assert(2 * kWaveRows * kFrequent <= kFreqSpace, "the rows' positions, listed and in order");
  rare_rows<T, G>(a, dout, (static_cast<int64_t>(blockIdx.x - a.freq_groups) * NW + wv) * kWaveRows, dtable,
                  reinterpret_cast<int32_t(*)[kFrequent]>(list[wv]), list[wv] + kWaveRows * kFrequent);
}

template <typename T, typename G>
void grad(GradArgs a, const void* dout, void* dtable, uint32_t* flags, hipStream_t st) {
  constexpr int kRows = kRowThreads / kWave * kWaveRows;
  // (777 tokens over 32,000 rows: clearing takes 4.8 of 65 us)
  a.table = a.n_tok <= kListTokens && static_cast<size_t>(a.V) * sizeof(RowList) >= kListSlots * sizeof(Distinct);
  if (a.table) {
    k_grad_list<true><<<1, kListTokens, 0, st>>>(a.s, a.tokens, a.n_tok, a.V, flags);
  } else {
    k_grad_clear<<<(static_cast<unsigned>(a.V) + 255) / 256, 256, 0, st>>>(a.s, a.V);
    if (a.n_tok > 0)
      k_grad_list<false><<<(static_cast<unsigned>(a.n_tok) + kListTokens - 1) / kListTokens, kListTokens, 0, st>>>(
          a.s, a.tokens, a.n_tok, a.V, flags);
  }
  a.freq_groups = a.n_tok > kFrequent ? kFreqGroups : 0;
  const unsigned blocks = static_cast<unsigned>(a.freq_groups) + (static_cast<unsigned>(a.V) + kRows - 1) / kRows;
  k_grad_rows<T, G><<<blocks, kRowThreads, 0, st>>>(a, static_cast<const T*>(dout), static_cast<G*>(dtable));
}

}  // namespace

hipError_t launch_embed_lookup(const void* table, int32_t V, int32_t d, fm_dtype dt, const int32_t* tokens, int32_t T,
                               float scale, void* out, uint32_t* flags, hipStream_t st) {
  if (dt == FM_BF16) lookup<uint16_t>(table, V, d, tokens, T, scale, out, flags, st);
  else lookup<float>(table, V, d, tokens, T, scale, out, flags, st);
  return hipGetLastError();
}

hipError_t launch_embed_pool(const void* table, int32_t V, int32_t d, fm_dtype dt, const int32_t* tokens, int32_t T,
                             const int32_t* offsets, int32_t B, float scale, uint16_t* out, uint32_t* flags,
                             hipStream_t st) {
  if (dt == FM_BF16) pool<uint16_t>(table, V, d, tokens, T, offsets, B, scale, out, flags, st);
  else pool<float>(table, V, d, tokens, T, offsets, B, scale, out, flags, st);
  return hipGetLastError();
}

size_t embed_grad_scratch_bytes(int32_t T, int32_t V) { return scratch_parts(T, V, nullptr, nullptr); }

hipError_t launch_embed_grad(const void* dout, fm_dtype dt, const int32_t* tokens, int32_t T, int32_t V, int32_t d,
                             float scale, bool accumulate, void* dtable, fm_dtype gdt, void* scratch, uint32_t* flags,
                             hipStream_t st) {
  GradArgs a;
  scratch_parts(T, V, &a.s, static_cast<char*>(scratch));
  a.tokens = tokens;
  a.n_tok = T;
  a.V = V;
  a.d = d;
  a.scale = scale;
  a.accumulate = accumulate;
  if (dt == FM_BF16 && gdt == FM_BF16) grad<uint16_t, uint16_t>(a, dout, dtable, flags, st);
  else if (dt == FM_BF16) grad<uint16_t, float>(a, dout, dtable, flags, st);
  else if (gdt == FM_BF16) grad<float, uint16_t>(a, dout, dtable, flags, st);
  else grad<float, float>(a, dout, dtable, flags, st);
  return hipGetLastError();
}

}  // namespace fm
