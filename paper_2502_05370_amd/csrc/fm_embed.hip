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

template <typename T>
struct Vec;   // 16 bytes of a row, aligned to an element only
template <>
struct Vec<uint16_t> {
  static constexpr int N = 8;
  typedef uint16_t raw __attribute__((ext_vector_type(8)));
  typedef raw mem __attribute__((aligned(2)));
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  typedef float raw __attribute__((ext_vector_type(4)));
  typedef raw mem __attribute__((aligned(4)));
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
template <typename T>
__device__ __forceinline__ typename Vec<T>::raw load_part(const T* p, int n) {
  typename Vec<T>::raw v = {};
  if (n >= Vec<T>::N) {
    v = *reinterpret_cast<const typename Vec<T>::mem*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < Vec<T>::N - 1; ++i)
      if (i < n) v[i] = p[i];
  }
  return v;
}
template <typename T>
__device__ __forceinline__ void store_part(T* p, typename Vec<T>::raw v, int n) {
  if (n >= Vec<T>::N) {
    *reinterpret_cast<typename Vec<T>::mem*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < Vec<T>::N - 1; ++i)
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
// row spans gridDim.y groups.
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
    store_part(dst + c, v[u], d - c);
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
// each XCD's L2 sees one eighth of the columns of the frequent rows.
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
    store_part(dst, v, have);
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
  const int nv = (d + Vec<T>::N - 1) / Vec<T>::N;
  auto blocks = [&](int cl) { return (nv + cl - 1) / cl; };
  if (static_cast<int64_t>(B) * blocks(32) >= 1024)
    pool_cl<T, 32>(table, V, d, tokens, T_, offsets, B, scale, out, flags, blocks(32), st);
  else
    pool_cl<T, 8>(table, V, d, tokens, T_, offsets, B, scale, out, flags, blocks(8), st);
}

// ---------------------------------------------------------------- gradient

// A frequent token's row (more than kFrequent tokens select it) is summed by
// whole workgroups, every other row by one wavefront.
constexpr int kFrequent = 32;
constexpr int kGradThreads = 256;
constexpr int kFreqThreads = 512;
constexpr int kFreqLanes = 32;      // lanes over the columns of a frequent row's block
constexpr int kFreqGroups = 512;    // workgroups that share the frequent rows
constexpr int kFreqList = 512;      // positions a wavefront lists at a time

struct GradScratch {
  int32_t* head;     // [V] last token listed for the row (-1: none)
  int32_t* count;    // [V] tokens of the row
  int32_t* next;     // [T] the token listed before it in its row
  int32_t* freq;     // [T / kFrequent] the frequent rows
  int32_t* n_freq;
};

size_t scratch_parts(int32_t T, int32_t V, GradScratch* s, char* base) {
  size_t o = 0;
  auto part = [&](size_t n, int32_t** p) {
    if (s != nullptr) *p = reinterpret_cast<int32_t*>(base + o);
    o += align_up(n * sizeof(int32_t), kAlign);
  };
  GradScratch dummy;
  GradScratch* g = s != nullptr ? s : &dummy;
  part(1, &g->n_freq);
  part(static_cast<size_t>(V), &g->head);
  part(static_cast<size_t>(V), &g->count);
  part(static_cast<size_t>(T), &g->next);
  part(static_cast<size_t>(T) / kFrequent + 1, &g->freq);
  return o;
}

__global__ void __launch_bounds__(256) k_grad_clear(GradScratch s, int32_t V) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i == 0) *s.n_freq = 0;
  if (i < V) {
    s.head[i] = -1;
    s.count[i] = 0;
  }
}

// Each row's tokens become a list in an order that depends on timing; the sums
// below put the positions back in order.
__global__ void __launch_bounds__(256) k_grad_list(GradScratch s, const int32_t* __restrict__ tokens, int32_t n_tok,
                                                   int32_t V, uint32_t* __restrict__ flags) {
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (t >= n_tok) return;
  const int row = row_of(tokens[t], V, flags);
  if (row < 0) return;
  s.next[t] = atomicExch(&s.head[row], static_cast<int32_t>(t));
  if (atomicAdd(&s.count[row], 1) == kFrequent) s.freq[atomicAdd(s.n_freq, 1)] = row;
}

template <typename G>
__device__ __forceinline__ void put_row(G* dst, const float* acc, int n, float scale, bool accumulate, bool any) {
  constexpr int N = Vec<G>::N;
  typename Vec<G>::raw v = {};
  if (accumulate) v = load_part(dst, n);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float s = any ? acc[i] * scale : 0.0f;
    v[i] = narrow<G>(accumulate ? widen(v[i]) + s : s);
  }
  store_part(dst, v, n);
}

// acc[N of T] (one 16-byte vector of dout) into dtable, whose vectors may be
// half or twice as long.
template <typename T, typename G>
__device__ __forceinline__ void put_vec(G* dst, const float* acc, int n, float scale, bool accumulate, bool any) {
  if constexpr (Vec<T>::N <= Vec<G>::N) {
    if constexpr (Vec<T>::N == Vec<G>::N) {
      put_row(dst, acc, n, scale, accumulate, any);
    } else {   // float rows into a bf16 table: half a vector
#pragma unroll
      for (int i = 0; i < Vec<T>::N; ++i) {
        if (i >= n) break;
        const float s = any ? acc[i] * scale : 0.0f;
        dst[i] = narrow<G>(accumulate ? widen(dst[i]) + s : s);
      }
    }
  } else {
    put_row(dst, acc, n, scale, accumulate, any);
    if (n > Vec<G>::N) put_row(dst + Vec<G>::N, acc + Vec<G>::N, n - Vec<G>::N, scale, accumulate, any);
  }
}

// Rows of at most kFrequent tokens, one wavefront each: the row's positions are
// read off its list, put in order by rank (each lane holds one), and the rows of
// dout added in that order.  Rows without a token are written as zeros, or left
// alone when accumulating.
template <typename T, typename G>
__device__ __forceinline__ void rare_row(const GradScratch& s, const T* __restrict__ dout, int32_t d, int64_t row,
                                         float scale, bool accumulate, G* __restrict__ dtable, int32_t* ord) {
  constexpr int N = Vec<T>::N;
  constexpr int U = 4;
  const int lane = threadIdx.x % kWave;
  const int n = s.count[row];
  if (n > kFrequent || (accumulate && n == 0)) return;
  if (n > 0) {
    int mine = s.head[row];
    if (n > 1) {
      int p = mine;
      for (int i = 1; i < n; ++i) {
        p = s.next[p];
        if (lane == i) mine = p;
      }
      int rank = 0;
      for (int i = 0; i < n; ++i) rank += __shfl(mine, i, kWave) < mine ? 1 : 0;
      if (lane < n) ord[rank] = mine;
    } else if (lane == 0) {
      ord[0] = mine;
    }
  }
  wait_lgkm0();
  G* dst = dtable + row * d;
  for (int c0 = lane * N; c0 < d; c0 += U * kWave * N) {
    float acc[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i) acc[u][i] = 0.0f;
    for (int j = 0; j < n; ++j) {
      const T* src = dout + static_cast<int64_t>(ord[j]) * d;
      typename Vec<T>::raw v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u * kWave * N;
        v[u] = load_part(src + c, d - c);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < N; ++i) acc[u][i] += widen(v[u][i]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * kWave * N;
      if (c < d) put_vec<T, G>(dst + c, acc[u], d - c, scale, accumulate, n > 0);
    }
  }
}

template <typename T, typename G>
__global__ void __launch_bounds__(kGradThreads) k_grad_rare(GradScratch s, const T* __restrict__ dout, int32_t V,
                                                            int32_t d, float scale, bool accumulate,
                                                            G* __restrict__ dtable) {
  __shared__ int32_t ord[kGradThreads / kWave][kFrequent];
  const int wv = threadIdx.x / kWave;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kGradThreads / kWave) + wv;
  if (row < V) rare_row<T, G>(s, dout, d, row, scale, accumulate, dtable, ord[wv]);
}

// Frequent rows: a workgroup takes (row, block of columns) units in turn.  Its
// wavefronts share the batch in equal ranges, list their tokens of the row in
// order, and each lane group adds every second listed row; the groups' and
// wavefronts' sums are joined in a fixed order.
template <typename T, typename G>
__global__ void __launch_bounds__(kFreqThreads) k_grad_frequent(GradScratch s, const T* __restrict__ dout,
                                                                const int32_t* __restrict__ tokens, int32_t n_tok,
                                                                int32_t d, float scale, bool accumulate,
                                                                G* __restrict__ dtable) {
  constexpr int N = Vec<T>::N;
  constexpr int NW = kFreqThreads / kWave;
  constexpr int GR = kWave / kFreqLanes;
  constexpr int U = 8;
  __shared__ int32_t list[NW][kFreqList + kWave];
  __shared__ float part[NW][kFreqLanes * N + 4];
  const int lane = threadIdx.x % kWave;
  const int wv = threadIdx.x / kWave;
  const int n_blk = (d + kFreqLanes * N - 1) / (kFreqLanes * N);
  const int64_t units = static_cast<int64_t>(*s.n_freq) * n_blk;
  const int share = (n_tok + NW * kWave - 1) / (NW * kWave) * kWave;   // tokens per wavefront
  const int first = wv * share;   // (n_tok + NW * kWave fits: the host bounds T)
  const int last = first + share < n_tok ? first + share : n_tok;
  for (int64_t u0 = blockIdx.x; u0 < units; u0 += gridDim.x) {
    const int32_t row = s.freq[u0 / n_blk];
    const int col = (static_cast<int>(u0 % n_blk) * kFreqLanes + lane % kFreqLanes) * N;
    const int have = d - col;
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.0f;
    int n = 0;   // listed positions
    auto drain = [&]() __attribute__((always_inline)) {
      wait_lgkm0();
      for (int i0 = lane / kFreqLanes; i0 < n; i0 += U * GR) {
        typename Vec<T>::raw v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + u * GR;
          v[u] = load_part(dout + static_cast<int64_t>(i < n ? list[wv][i] : 0) * d + col, i < n ? have : 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < N; ++i) acc[i] += widen(v[u][i]);
      }
      n = 0;
    };
    for (int t = first; t < last; t += kWave) {
      const bool hit = t + lane < last && tokens[t + lane] == row;
      const uint64_t m = __ballot(hit);
      if (m == 0) continue;
      if (hit) list[wv][n + __popcll(m & ((1ull << lane) - 1ull))] = t + lane;
      n += __popcll(m);
      if (n >= kFreqList) drain();
    }
    drain();
#pragma unroll
    for (int m = kFreqLanes; m < kWave; m <<= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] += __shfl_xor(acc[i], m, kWave);
    if (lane < kFreqLanes)
#pragma unroll
      for (int i = 0; i < N; ++i) part[wv][lane * N + i] = acc[i];
    __syncthreads();
    if (wv == 0 && lane < kFreqLanes && have > 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        acc[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) acc[i] += part[w][lane * N + i];
      }
      put_vec<T, G>(dtable + static_cast<int64_t>(row) * d + col, acc, have, scale, accumulate, true);
    }
    __syncthreads();
  }
}

template <typename T, typename G>
void grad(const void* dout, const int32_t* tokens, int32_t n_tok, int32_t V, int32_t d, float scale, bool accumulate,
          void* dtable, const GradScratch& s, uint32_t* flags, hipStream_t st) {
  k_grad_clear<<<(static_cast<unsigned>(V) + 255) / 256, 256, 0, st>>>(s, V);
  if (n_tok > 0) k_grad_list<<<(static_cast<unsigned>(n_tok) + 255) / 256, 256, 0, st>>>(s, tokens, n_tok, V, flags);
  if (n_tok > kFrequent)
    k_grad_frequent<T, G><<<kFreqGroups, kFreqThreads, 0, st>>>(s, static_cast<const T*>(dout), tokens, n_tok, d, scale,
                                                                accumulate, static_cast<G*>(dtable));
  constexpr int kRows = kGradThreads / kWave;
  k_grad_rare<T, G><<<(static_cast<unsigned>(V) + kRows - 1) / kRows, kGradThreads, 0, st>>>(
      s, static_cast<const T*>(dout), V, d, scale, accumulate, static_cast<G*>(dtable));
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
  GradScratch s;
  scratch_parts(T, V, &s, static_cast<char*>(scratch));
  if (dt == FM_BF16 && gdt == FM_BF16) grad<uint16_t, uint16_t>(dout, tokens, T, V, d, scale, accumulate, dtable, s, flags, st);
  else if (dt == FM_BF16) grad<uint16_t, float>(dout, tokens, T, V, d, scale, accumulate, dtable, s, flags, st);
  else if (gdt == FM_BF16) grad<float, uint16_t>(dout, tokens, T, V, d, scale, accumulate, dtable, s, flags, st);
  else grad<float, float>(dout, tokens, T, V, d, scale, accumulate, dtable, s, flags, st);
  return hipGetLastError();
}

}  // namespace fm
