// Pages of the key-value cache: who holds them (resize, fork, compact), their
// contents (copy) and the rows of new tokens (write, read).
//
// Bookkeeping is integers: one workgroup decides (or one per slot, where
// decisions are apart), and a second launch moves pages, whose list the first
// wrote.  Counts change by atomics, whose order does not matter.
//
// Memory bounds what moves, launches what decides.  Compacting a pool half of whose 1,057
// pages of 1.6 MB live, 264 of them moved: 4.7 us to decide, 157 to move (831 MB, 5.3
// TB/s; a copy reaches 5.1).  Eight slots forked in four, each grown past a shared page:
// 2.3 us of new tables, 1.7 to put them in place, 7.0 to decide, 15 to copy 32 pages (100
// MB, 6.6 TB/s: the memory-side cache holds some).  Rows of 8,192 tokens on 8 heads of 128
// bf16, which the caches hold since they were made: 67 MB in 18 us (3.7 TB/s), from
// memory 26; of 8 tokens 3.3 us.
//
// One workgroup decides for a pool of any size, reading its counts: growth takes 9 us
// up to a thousand pages, 41 in one of 131,072 whose free pages are the last, 267 and
// 4,300 of 2^20 and 2^24; a compaction that moves nothing 11, 102, 974 and 15,700.
// (131,072 pages of 2.2 MB are 288 GB.)
#include "fm_device.h"
#include "fm_kv.h"

namespace fm {

namespace {

constexpr int kPlan = 1024;                  // threads of a deciding workgroup
constexpr int kPlanWaves = kPlan / kWave;
constexpr int kMoveThreads = 256;
constexpr int kMoveGrid = 1024;
constexpr int kMoveBytes = kMoveThreads * 16 * 4;   // of one workgroup's turn

// Scratch of a call, its parts 256-byte aligned.
struct Scratch {
  int32_t* count;   // [0]: pages to move
  int32_t* src;     // [max(n_slots, n_pages)] pages to move
  int32_t* dst;     //   and where to
  int32_t* need;    // [n_slots] new pages of a slot; fork: its new length
  int32_t* start;   // [n_slots] new pages of the slots before it
  int32_t* list;    // [n_pages] free pages; compact: new page numbers; copy: how often a page is named
  int32_t* rows;    // [n_slots][max_pages] fork: the tables to come
  size_t bytes;
};

Scratch carve(char* base, const fm_kv_cache& c) {
  Scratch s{};
  size_t at = 0;
  auto take = [&](size_t n) {
    int32_t* p = reinterpret_cast<int32_t*>(base + at);
    at += align_up(n * sizeof(int32_t), kAlign);
    return p;
  };
  const size_t moves = static_cast<size_t>(c.n_slots > c.n_pages ? c.n_slots : c.n_pages);
  s.count = take(1);
  s.src = take(moves);
  s.dst = take(moves);
  s.need = take(static_cast<size_t>(c.n_slots));
  s.start = take(static_cast<size_t>(c.n_slots));
  s.list = take(static_cast<size_t>(c.n_pages));
  s.rows = take(static_cast<size_t>(c.n_slots) * static_cast<size_t>(c.max_pages));
  s.bytes = at;
  return s;
}

__device__ __forceinline__ void set_flags(uint32_t* flags, uint32_t bits) {
  if (flags != nullptr) atomicOr(flags, bits);
}

// What the workgroup wrote is in the L2, and plain loads of its wavefronts see it:
// they share a first cache.  Words that atomics changed are read past that cache
// (`count_of`); a fence of the device's scope, which writes the L2 back, is not needed
// by a single workgroup.
__device__ __forceinline__ void settle() {
  wait_vmcnt<0>();
  __syncthreads();
}
__device__ __forceinline__ int32_t count_of(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ int64_t wave_scan(int64_t v) {   // inclusive
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const int64_t o = __shfl_up(v, m, kWave);
    if (lane >= m) v += o;
  }
  return v;
}

// Sum of v over the threads before this one; *total over all.  sums: kPlanWaves
// values of LDS, free again after the next barrier of the caller.
__device__ __forceinline__ int64_t plan_scan(int64_t v, int64_t* sums, int64_t* total) {
  const int lane = threadIdx.x % kWave;
  const int wv = threadIdx.x / kWave;
  const int64_t upto = wave_scan(v);
  __syncthreads();
  if (lane == kWave - 1) sums[wv] = upto;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const int64_t s = sums[w];
    before += w < wv ? s : 0;
    all += s;
  }
  *total = all;
  return before + upto - v;
}

constexpr int kFew = 4;                // new pages that a lane hands out by itself
constexpr int32_t kRefused = -1;       // need of a slot that does not grow, or must not
constexpr int32_t kCopies = 1 << 30;   // bit of a slot whose last page is copied

// One workgroup.  Slots drop tokens, then needs are counted, the lowest free
// pages listed until they suffice, and handed out.
__global__ void __launch_bounds__(kPlan) k_kv_resize(KvArgs a, const int32_t* delta, uint8_t* granted, uint32_t* flags,
                                                     Scratch sc) {
  __shared__ int64_t sums[kPlanWaves];
  __shared__ int32_t moves;
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  if (tid == 0) moves = 0;
  uint32_t bad = 0;

  // drop: a wavefront per slot that does
  for (int s0 = 0; s0 < a.n_slots; s0 += kWave) {
    const int mine = s0 + lane < a.n_slots ? delta[s0 + lane] : 0;
    uint64_t todo = __ballot(mine < 0);
    for (int k = 0; todo != 0; ++k, todo &= todo - 1) {
      if (k % kPlanWaves != wv) continue;
      const int i = __builtin_ctzll(todo);
      const int s = s0 + i;
      const int32_t len = a.tokens(a.length[s]);
      const int64_t left = static_cast<int64_t>(len) + __builtin_amdgcn_readlane(mine, i);
      const int32_t end = left > 0 ? static_cast<int32_t>(left) : 0;
      const int32_t n1 = a.pages_of(len);
      for (int p = a.pages_of(end) + lane; p < n1; p += kWave) {
        int32_t* entry = a.table + static_cast<int64_t>(s) * a.max_pages + p;
        if (a.valid(*entry)) atomicSub(&a.refs[*entry], 1);
        else bad = FM_FLAG_INDEX_RANGE;
        *entry = -1;
      }
      if (lane == 0) a.length[s] = end;
    }
  }
  settle();

  // needs, in order of the slots
  int64_t before = 0;
  for (int s0 = 0; s0 < a.n_slots; s0 += kPlan) {
    const int s = s0 + tid;
    int32_t need = kRefused;
    if (s < a.n_slots && delta[s] > 0) {
      const int32_t len = a.tokens(a.length[s]);
      const int64_t end = static_cast<int64_t>(len) + delta[s];
      if (end > a.capacity()) {
        bad |= FM_FLAG_PAGES_FULL;
      } else {
        need = a.pages_of(static_cast<int32_t>(end)) - a.pages_of(len);
        if (len % a.page != 0) {
          const int32_t last = a.table[static_cast<int64_t>(s) * a.max_pages + a.pages_of(len) - 1];
          if (!a.valid(last)) {
            bad |= FM_FLAG_INDEX_RANGE;
            need = kRefused;
          } else if (count_of(&a.refs[last]) > 1) {
            need = (need + 1) | kCopies;
          }
        }
      }
    }
    int64_t all;
    const int64_t ahead = plan_scan(need == kRefused ? 0 : need & ~kCopies, sums, &all);
    if (s < a.n_slots) {
      sc.need[s] = need;
      // (a prefix past all pages is as good as one page past them)
      sc.start[s] = static_cast<int32_t>(before + ahead <= a.n_pages ? before + ahead : a.n_pages + 1);
    }
    before += all;
  }

  // the lowest free pages, as many as are needed
  const int64_t wanted = before;
  int64_t found = 0;
  for (int p0 = 0; p0 < a.n_pages && found < wanted; p0 += kPlan * 4) {
    bool is_free[4];
    int n = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = p0 + tid * 4 + j;
      is_free[j] = p < a.n_pages && count_of(&a.refs[p]) == 0;
      n += is_free[j] ? 1 : 0;
    }
    int64_t all;
    int64_t at = found + plan_scan(n, sums, &all);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (is_free[j]) sc.list[at++] = p0 + tid * 4 + j;
    found += all;
  }
  settle();

  // handed out: by a lane per slot up to kFew pages, beyond by a wavefront
  auto pages_of_need = [&](int32_t need) __attribute__((always_inline)) {
    return need == kRefused ? 0 : need & ~kCopies;
  };
  // entry j of the new ones in a slot's row
  auto hand = [&](int32_t* row, int first, int copies, int j) __attribute__((always_inline)) {
    const int32_t p = sc.list[first + j];
    if (j < copies) {   // the shared page's copy takes its place
      const int32_t old = row[j];
      const int at = atomicAdd(&moves, 1);
      sc.src[at] = old;
      sc.dst[at] = p;
      atomicSub(&a.refs[old], 1);
    }
    row[j] = p;
    a.refs[p] = 1;
  };
  for (int s = tid; s < a.n_slots; s += kPlan) {
    const int32_t need = sc.need[s];
    const int32_t start = sc.start[s];
    const int32_t pages = pages_of_need(need);
    const bool grows = need != kRefused && (pages == 0 || static_cast<int64_t>(start) + pages <= found);
    if (need != kRefused && !grows) bad |= FM_FLAG_PAGES_FULL;
    if (granted != nullptr) granted[s] = grows ? 1 : 0;
    if (!grows || pages > kFew) continue;
    const int32_t len = a.tokens(a.length[s]);
    const int copies = (need & kCopies) != 0 ? 1 : 0;
    int32_t* row = a.table + static_cast<int64_t>(s) * a.max_pages + a.pages_of(len) - copies;
    for (int j = 0; j < pages; ++j) hand(row, start, copies, j);
    a.length[s] = len + delta[s];
  }
  for (int s0 = 0; s0 < a.n_slots; s0 += kWave) {
    const int s = s0 + lane;
    const int32_t need = s < a.n_slots ? sc.need[s] : kRefused;
    const int32_t start = s < a.n_slots ? sc.start[s] : 0;
    const int32_t pages = pages_of_need(need);
    uint64_t todo = __ballot(pages > kFew && static_cast<int64_t>(start) + pages <= found);
    for (int k = 0; todo != 0; ++k, todo &= todo - 1) {
      if (k % kPlanWaves != wv) continue;
      const int i = __builtin_ctzll(todo);
      const int n = __builtin_amdgcn_readlane(pages, i);
      const int first = __builtin_amdgcn_readlane(start, i);
      const int copies = (__builtin_amdgcn_readlane(need, i) & kCopies) != 0 ? 1 : 0;
      const int32_t len = a.tokens(a.length[s0 + i]);
      int32_t* row = a.table + static_cast<int64_t>(s0 + i) * a.max_pages + a.pages_of(len) - copies;
      for (int j = lane; j < n; j += kWave) hand(row, first, copies, j);
      if (lane == 0) a.length[s0 + i] = len + delta[s0 + i];
    }
  }
  if (bad != 0) set_flags(flags, bad);
  __syncthreads();
  if (tid == 0) *sc.count = moves;
}

// Pages to their new places.  With `names`, the entries of the tables follow.
__global__ void __launch_bounds__(kMoveThreads) k_kv_move(KvArgs a, Scratch sc, const int32_t* names) {
  const int n = *sc.count;
  const int turns = static_cast<int>((a.page_bytes + kMoveBytes - 1) / kMoveBytes);   // of a page
  const int64_t all = static_cast<int64_t>(n) * turns;
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const int m = static_cast<int>(u / turns);
    const int64_t at = (u % turns) * kMoveBytes + threadIdx.x * 16;
    const char* from = a.pages + sc.src[m] * a.page_bytes;
    char* to = a.pages + sc.dst[m] * a.page_bytes;
    uint32x4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at + j * kMoveThreads * 16 < a.page_bytes)
        v[j] = __builtin_nontemporal_load(reinterpret_cast<const uint32x4*>(from + at + j * kMoveThreads * 16));
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at + j * kMoveThreads * 16 < a.page_bytes)
        __builtin_nontemporal_store(v[j], reinterpret_cast<uint32x4*>(to + at + j * kMoveThreads * 16));
  }
  if (names != nullptr) {
    const int64_t entries = static_cast<int64_t>(a.n_slots) * a.max_pages;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kMoveThreads + threadIdx.x; i < entries;
         i += static_cast<int64_t>(gridDim.x) * kMoveThreads) {
      const int32_t p = a.table[i];
      if (a.valid(p) && names[p] != p) a.table[i] = names[p];
    }
  }
}

// A slot per workgroup: the table it will have, beside the present ones, which
// others still read, and the counts of the pages it takes and gives back.
__global__ void __launch_bounds__(256) k_kv_fork_take(KvArgs a, const int32_t* parent, uint32_t* flags, Scratch sc) {
  const int s = blockIdx.x;
  const int p = parent[s];
  const bool stays = p < 0 || p >= a.n_slots || p == s;
  const int32_t len = stays ? 0 : a.tokens(a.length[p]);
  uint32_t bad = p >= a.n_slots ? FM_FLAG_INDEX_RANGE : 0u;
  if (threadIdx.x == 0) sc.need[s] = stays ? -1 : len;
  if (!stays) {
    const int32_t* from = a.table + static_cast<int64_t>(p) * a.max_pages;
    const int32_t* own = a.table + static_cast<int64_t>(s) * a.max_pages;
    int32_t* row = sc.rows + static_cast<int64_t>(s) * a.max_pages;
    const int n = a.pages_of(len);
    for (int i = threadIdx.x; i < n; i += 256) {
      const int32_t e = from[i];
      row[i] = e;
      if (a.valid(e)) atomicAdd(&a.refs[e], 1);
      else bad = FM_FLAG_INDEX_RANGE;
    }
    const int n0 = a.pages_of(a.tokens(a.length[s]));
    for (int i = threadIdx.x; i < n0; i += 256) {
      const int32_t e = own[i];
      if (a.valid(e)) atomicSub(&a.refs[e], 1);
      else bad = FM_FLAG_INDEX_RANGE;
    }
  }
  if (bad != 0) set_flags(flags, bad);
}

__global__ void __launch_bounds__(256) k_kv_fork_put(KvArgs a, Scratch sc) {
  const int s = blockIdx.x;
  const int32_t len = sc.need[s];
  if (len < 0) return;
  const int n0 = a.pages_of(a.tokens(a.length[s]));
  const int n = a.pages_of(len);
  int32_t* own = a.table + static_cast<int64_t>(s) * a.max_pages;
  const int32_t* row = sc.rows + static_cast<int64_t>(s) * a.max_pages;
  for (int i = threadIdx.x; i < (n > n0 ? n : n0); i += 256) own[i] = i < n ? row[i] : -1;
  __syncthreads();   // all have read the old length
  if (threadIdx.x == 0) a.length[s] = len;
}

// Small tables in one launch: a workgroup holds all entries in registers between
// reading and writing them.  40 slots of 34 entries 3.7 us, 5.0 in two launches (calls
// one after another 5.6 and 8.4); 64 of 64, four entries a thread, 6.7 and 5.0.
constexpr int kForkEach = 2;   // entries of a thread
__global__ void __launch_bounds__(kPlan) k_kv_fork(KvArgs a, const int32_t* parent, uint32_t* flags) {
  const int entries = a.n_slots * a.max_pages;
  uint32_t bad = 0;
  int p[kForkEach], own[kForkEach], len[kForkEach], old[kForkEach], to[kForkEach];
#pragma unroll
  for (int k = 0; k < kForkEach; ++k) {
    const int i = static_cast<int>(threadIdx.x) + k * kPlan;
    p[k] = i < entries ? parent[i / a.max_pages] : -1;
    own[k] = i < entries ? a.length[i / a.max_pages] : 0;
    old[k] = i < entries ? a.table[i] : 0;
  }
#pragma unroll
  for (int k = 0; k < kForkEach; ++k) {
    const int i = static_cast<int>(threadIdx.x) + k * kPlan;
    if (p[k] >= a.n_slots) bad = FM_FLAG_INDEX_RANGE;
    if (p[k] >= a.n_slots || p[k] == i / a.max_pages) p[k] = -1;
    const int from = p[k] < 0 ? 0 : p[k];
    len[k] = a.tokens(a.length[from]);
    to[k] = a.table[static_cast<int64_t>(from) * a.max_pages + i % a.max_pages];
  }
  settle();
#pragma unroll
  for (int k = 0; k < kForkEach; ++k) {
    if (p[k] < 0) continue;
    const int i = static_cast<int>(threadIdx.x) + k * kPlan;
    const int j = i % a.max_pages;
    const bool had = j < a.pages_of(a.tokens(own[k])), has = j < a.pages_of(len[k]);
    if (had) {
      if (a.valid(old[k])) atomicSub(&a.refs[old[k]], 1);
      else bad = FM_FLAG_INDEX_RANGE;
    }
    if (has) {
      if (a.valid(to[k])) atomicAdd(&a.refs[to[k]], 1);
      else bad = FM_FLAG_INDEX_RANGE;
    }
    if (had || has) a.table[i] = has ? to[k] : -1;
    if (j == 0) a.length[i / a.max_pages] = len[k];
  }
  if (bad != 0) set_flags(flags, bad);
}

// One workgroup: how many pages live, then the live ones from there on and the
// free ones before it, both in order and as many of each.
__global__ void __launch_bounds__(kPlan) k_kv_compact(KvArgs a, int32_t* live_out, Scratch sc) {
  __shared__ int64_t sums[kPlanWaves];
  const int tid = threadIdx.x;
  int64_t mine = 0, live;
  for (int p = tid; p < a.n_pages; p += kPlan) mine += a.refs[p] > 0 ? 1 : 0;
  plan_scan(mine, sums, &live);
  int64_t sources = 0, holes = 0;
  for (int p0 = 0; p0 < a.n_pages; p0 += kPlan * 4) {
    int kind[4];   // 1: a source, 2: a hole
    int64_t n = 0;   // sources in the lower half, holes in the upper
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = p0 + tid * 4 + j;
      const bool held = p < a.n_pages && a.refs[p] > 0;
      kind[j] = p >= a.n_pages ? 0 : (held && p >= live ? 1 : (!held && p < live ? 2 : 0));
      n += kind[j] == 1 ? 1 : (kind[j] == 2 ? int64_t{1} << 32 : 0);
    }
    int64_t all;
    const int64_t at = plan_scan(n, sums, &all);
    int64_t is = sources + (at & 0xFFFFFFFF), ih = holes + (at >> 32);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = p0 + tid * 4 + j;
      if (kind[j] == 1) sc.src[is++] = p;
      if (kind[j] == 2) sc.dst[ih++] = p;
      if (p < a.n_pages) sc.list[p] = p;
    }
    sources += all & 0xFFFFFFFF;
    holes += all >> 32;
  }
  settle();
  for (int i = tid; i < sources; i += kPlan) {
    const int32_t from = sc.src[i], to = sc.dst[i];
    sc.list[from] = to;
    a.refs[to] = a.refs[from];
    a.refs[from] = 0;
  }
  if (tid == 0) {
    *sc.count = static_cast<int32_t>(sources);
    if (live_out != nullptr) *live_out = static_cast<int32_t>(live);
  }
}

// One workgroup: pairs that can be copied side by side, in any order.
__global__ void __launch_bounds__(kPlan) k_kv_pairs(KvArgs a, const int32_t* src, const int32_t* dst, int32_t n,
                                                    uint32_t* flags, Scratch sc) {
  __shared__ int32_t kept;
  const int tid = threadIdx.x;
  if (tid == 0) kept = 0;
  for (int i = tid; i < n; i += kPlan) {
    if (a.valid(src[i])) sc.list[src[i]] = 0;
    if (a.valid(dst[i])) sc.list[dst[i]] = 0;
  }
  settle();
  for (int i = tid; i < n; i += kPlan) {
    if (a.valid(src[i])) atomicAdd(&sc.list[src[i]], 1);
    if (a.valid(dst[i])) atomicAdd(&sc.list[dst[i]], 1);
  }
  settle();
  for (int i = tid; i < n; i += kPlan) {
    const int32_t s = src[i], d = dst[i];
    const bool fits = a.valid(s) && a.valid(d) &&
                      count_of(&sc.list[d]) == 1;
    if (!fits) {
      set_flags(flags, FM_FLAG_INDEX_RANGE);
      continue;
    }
    const int at = atomicAdd(&kept, 1);
    sc.src[at] = s;
    sc.dst[at] = d;
  }
  __syncthreads();
  if (tid == 0) *sc.count = kept;
}

// ---------------------------------------------------------------- rows

constexpr int kRowWaves = 4;

// The new tokens of a slot: places [p0, p1) of its sequence, p0's row is `row`.
struct Span {
  int32_t p0, p1, row;
  __device__ __forceinline__ int blocks() const {
    return p1 > p0 ? (p1 + kBlockTokens - 1) / kBlockTokens - p0 / kBlockTokens : 0;
  }
};

__device__ __forceinline__ Span span_of(const KvArgs& a, const KvRows& r, int s, uint32_t& bad) {
  const int32_t len = a.tokens(a.length[s]);
  Span w{0, 0, 0};
  if (r.active != nullptr && r.active[s] == 0) return w;
  int32_t n = 1, row = s;
  if (r.offsets != nullptr) {
    const int32_t lo = r.offsets[s], hi = r.offsets[s + 1];
    row = lo < 0 ? 0 : (lo < r.T ? lo : r.T);
    const int32_t end = hi < 0 ? 0 : (hi < r.T ? hi : r.T);
    n = end > row ? end - row : 0;
    if (n > len) {
      bad |= FM_FLAG_INDEX_RANGE;
      return w;
    }
  } else if (len == 0) {
    return w;
  }
  return Span{len - n, len, row};
}

// One piece of a block of one head, a wavefront.  Keys: lane 16 g + c has 16 bytes of
// token c.  Values: four tokens' columns; loads of single elements from 16
// neighbouring columns, so that a piece is stored whole where its tokens are all new.
template <typename T>
struct Piece {
  static constexpr int N = 16 / static_cast<int>(sizeof(T));   // elements of a lane
  uint32x4 k;
  alignas(16) T v[N];
  T* krow;        // this lane's places in the rows
  T* vrow;
  int d;          // first dimension of the lane's keys
  bool has, quad[4];
  __device__ __forceinline__ Piece(const KvArgs& a, const KvRows& r, const Span& w, int pos0, int head, int piece) {
    const int lane = threadIdx.x % kWave;
    const int c = lane % 16, g = lane / 16;
    d = 4 * N * piece + N * g;
    has = pos0 + c >= w.p0 && pos0 + c < w.p1;
    const int64_t col0 = static_cast<int64_t>(head) * a.head_dim;
    krow = static_cast<T*>(r.k) + (w.row + (pos0 + c - w.p0)) * r.k_stride + col0 + d;
    // token 4 g of the block; rows outside the span are not touched
    vrow = static_cast<T*>(r.v) + (w.row + (pos0 + 4 * g - w.p0)) * r.v_stride + col0 + 4 * N * piece + c;
#pragma unroll
    for (int j = 0; j < 4; ++j) quad[j] = pos0 + 4 * g + j >= w.p0 && pos0 + 4 * g + j < w.p1;
  }
  // whether column 16 i + c of the piece is one of the head's
  static __device__ __forceinline__ bool column(const KvArgs& a, int piece, int i) {
    return 4 * N * piece + 16 * i + static_cast<int>(threadIdx.x % 16) < a.head_dim;
  }
  __device__ __forceinline__ void from_rows(const KvArgs& a, const KvRows& r, int piece) {
    k = uint32x4{0u, 0u, 0u, 0u};
    if (has && d < a.head_dim) k = *reinterpret_cast<const uint32x4*>(krow);
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[4 * i + j] = T(0);
        if (quad[j] && column(a, piece, i)) v[4 * i + j] = vrow[j * r.v_stride + 16 * i];
      }
  }
  // MANY: past the caches, which many rows would turn over: 8,192 tokens of 8 heads of 128
  // bf16 to pages that no cache holds 17.6 us, 19.2 through them (26 and 29 where the
  // rows come from memory too); one token of each of 256 slots, 32 heads of 128, 15.8
  // and 16.2, float32 20.7 and 25.0.  A few tokens stay there for the attention that
  // follows.
  template <bool MANY>
  __device__ __forceinline__ void to_page(char* kp, char* vp) const {
    auto store = [](uint32x4 x, uint32x4* p) __attribute__((always_inline)) {
      if constexpr (MANY) __builtin_nontemporal_store(x, p);
      else *p = x;
    };
    const int lane = threadIdx.x % kWave;
    if (has) store(k, reinterpret_cast<uint32x4*>(kp) + lane);
    if (quad[0] && quad[3]) {
      store(*reinterpret_cast<const uint32x4*>(v), reinterpret_cast<uint32x4*>(vp) + lane);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (quad[e % 4]) reinterpret_cast<T*>(vp)[lane * N + e] = v[e];
    }
  }
  __device__ __forceinline__ void from_page(const char* kp, const char* vp) {
    const int lane = threadIdx.x % kWave;
    k = reinterpret_cast<const uint32x4*>(kp)[lane];
    *reinterpret_cast<uint32x4*>(v) = reinterpret_cast<const uint32x4*>(vp)[lane];
  }
  __device__ __forceinline__ void to_rows(const KvArgs& a, const KvRows& r, int piece) const {
    if (has && d < a.head_dim) *reinterpret_cast<uint32x4*>(krow) = k;
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (quad[j] && column(a, piece, i)) vrow[j * r.v_stride + 16 * i] = v[4 * i + j];
  }
};

// A workgroup takes blocks of 16 tokens; blocks are counted through the slots
// (each workgroup sums the slots' counts until it finds its own), the pieces of all
// heads are dealt to the wavefronts and to grid.y.
template <typename T, bool READ, bool MANY>
__global__ void __launch_bounds__(kRowWaves* kWave) k_kv_rows(KvArgs a, KvRows r) {
  constexpr int NT = kRowWaves * kWave;
  __shared__ int32_t sums[kRowWaves];
  __shared__ int32_t where[2];   // slot and block of it
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  uint32_t bad = 0;
  int64_t unit = blockIdx.x;
  int64_t total = 0;   // blocks of all slots, where this workgroup counts them all
  for (;;) {
    int slot = static_cast<int>(unit), block = 0;
    if (r.offsets != nullptr) {
      int64_t before = 0;
      if (tid == 0) where[0] = -1;
      for (int s0 = 0; s0 < a.n_slots; s0 += NT) {
        uint32_t range = 0;
        const int n = s0 + tid < a.n_slots ? span_of(a, r, s0 + tid, range).blocks() : 0;
        if (unit == 0 && blockIdx.y == 0) bad |= range;
        int upto = n;   // (of one turn: 256 slots of up to 2^20 blocks)
#pragma unroll
        for (int m = 1; m < kWave; m <<= 1) {
          const int o = __shfl_up(upto, m, kWave);
          if (lane >= m) upto += o;
        }
        __syncthreads();
        if (lane == kWave - 1) sums[wv] = upto;
        __syncthreads();
        int64_t at = before + upto - n;
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) {
          at += w < wv ? sums[w] : 0;
          before += sums[w];
        }
        if (unit >= at && unit < at + n) {
          where[0] = s0 + tid;
          where[1] = static_cast<int32_t>(unit - at);
        }
        if (before > unit && unit != 0) break;
      }
      __syncthreads();
      slot = __builtin_amdgcn_readfirstlane(where[0]);
      block = __builtin_amdgcn_readfirstlane(where[1]);
      if (unit == 0) total = before;
      __syncthreads();   // `where` may change again
    }
    if (slot >= 0) {
      uint32_t seen = 0;
      const Span w = span_of(a, r, slot, seen);
      if (w.p1 > w.p0) {
        const int pos0 = (w.p0 / kBlockTokens + block) * kBlockTokens;
        const int64_t at = static_cast<int64_t>(pos0 % a.page) * (a.pieces * kRowPiece);
        const int all = a.heads * a.pieces;
        const int32_t page = a.table[static_cast<int64_t>(slot) * a.max_pages + pos0 / a.page];
        const bool valid = a.valid(page);
        const bool shared = !READ && a.refs[valid ? page : 0] > 1;
        if (!valid) bad |= FM_FLAG_INDEX_RANGE;
        else if (shared) bad |= FM_FLAG_PAGE_SHARED;
        char* base = a.pages + (valid ? page : 0) * a.page_bytes + at;
        for (int i = static_cast<int>(blockIdx.y) * kRowWaves + wv; i < all; i += gridDim.y * kRowWaves) {
          const int head = i / a.pieces, piece = i % a.pieces;
          char* kp = base + a.head_offset(r.layer, 0, head) + piece * kPieceBytes;
          char* vp = base + a.head_offset(r.layer, 1, head) + piece * kPieceBytes;
          Piece<T> p(a, r, w, pos0, head, piece);
          if constexpr (READ) {
            if (!valid) break;
            p.from_page(kp, vp);
            p.to_rows(a, r, piece);
          } else {
            p.from_rows(a, r, piece);   // (on their way while the table's entry is)
            if (valid && !shared) p.template to_page<MANY>(kp, vp);
          }
        }
      }
    }
    // The grid has a workgroup for every block of ascending offsets.  Spans that
    // overlap have more: the first workgroup, which has counted them, takes those.
    if (blockIdx.x != 0) break;
    unit = unit == 0 ? gridDim.x : unit + 1;
    if (unit >= total) break;
  }
  if (bad != 0) set_flags(r.flags, bad);
}

void move(const KvArgs& a, const Scratch& sc, const int32_t* names, hipStream_t st) {
  k_kv_move<<<kMoveGrid, kMoveThreads, 0, st>>>(a, sc, names);
}

}  // namespace

size_t kv_scratch_bytes(const fm_kv_cache& c) { return carve(nullptr, c).bytes; }

hipError_t launch_kv_resize(const fm_kv_cache& c, const int32_t* delta, uint8_t* granted, uint32_t* flags,
                            void* scratch, hipStream_t st) {
  const KvArgs a = kv_args(c);
  const Scratch sc = carve(static_cast<char*>(scratch), c);
  k_kv_resize<<<1, kPlan, 0, st>>>(a, delta, granted, flags, sc);
  move(a, sc, nullptr, st);
  return hipGetLastError();
}

hipError_t launch_kv_fork(const fm_kv_cache& c, const int32_t* parent, uint32_t* flags, void* scratch,
                          hipStream_t st) {
  const KvArgs a = kv_args(c);
  const Scratch sc = carve(static_cast<char*>(scratch), c);
  if (static_cast<int64_t>(c.n_slots) * c.max_pages <= kForkEach * kPlan) {
    k_kv_fork<<<1, kPlan, 0, st>>>(a, parent, flags);
  } else {
    k_kv_fork_take<<<static_cast<unsigned>(c.n_slots), 256, 0, st>>>(a, parent, flags, sc);
    k_kv_fork_put<<<static_cast<unsigned>(c.n_slots), 256, 0, st>>>(a, sc);
  }
  return hipGetLastError();
}

hipError_t launch_kv_compact(const fm_kv_cache& c, int32_t* live, uint32_t* flags, void* scratch, hipStream_t st) {
  const KvArgs a = kv_args(c);
  const Scratch sc = carve(static_cast<char*>(scratch), c);
  k_kv_compact<<<1, kPlan, 0, st>>>(a, live, sc);
  move(a, sc, sc.list, st);
  return hipGetLastError();
}

hipError_t launch_kv_copy(const fm_kv_cache& c, const int32_t* src, const int32_t* dst, int32_t n, uint32_t* flags,
                          void* scratch, hipStream_t st) {
  const KvArgs a = kv_args(c);
  const Scratch sc = carve(static_cast<char*>(scratch), c);
  k_kv_pairs<<<1, kPlan, 0, st>>>(a, src, dst, n, flags, sc);
  move(a, sc, nullptr, st);
  return hipGetLastError();
}

hipError_t launch_kv_rows(const fm_kv_cache& c, const KvRows& r, bool read, hipStream_t st) {
  const KvArgs a = kv_args(c);
  // a slot's rows lie in at most n / 16 + 2 blocks
  const int64_t most = r.offsets == nullptr
                           ? c.n_slots
                           : r.T / kBlockTokens + 2 * static_cast<int64_t>(c.n_slots < r.T ? c.n_slots : r.T);
  // Pieces of a wavefront: one where the batch is small, or four, so that fewer
  // workgroups look for their block (us of 1 and 4, 8 heads of 128 bf16: 8 tokens 3.3
  // and 5.1, 4,096, which are 9,216 pieces, 14.5 and 15.5, 8,192, 17,408 pieces, 21.1 and
  // 17.6; reading those 21.3 and 18.5).
  const int64_t pieces = static_cast<int64_t>(c.heads) * a.pieces;
  const bool many = most * pieces >= 16384;
  const int64_t per_group = kRowWaves * (many ? 4 : 1);
  const dim3 grid(static_cast<unsigned>(most), static_cast<unsigned>((pieces + per_group - 1) / per_group));
  auto go = [&](auto t) {
    using T = decltype(t);
    if (read) k_kv_rows<T, true, false><<<grid, kRowWaves * kWave, 0, st>>>(a, r);
    else if (many) k_kv_rows<T, false, true><<<grid, kRowWaves * kWave, 0, st>>>(a, r);
    else k_kv_rows<T, false, false><<<grid, kRowWaves * kWave, 0, st>>>(a, r);
  };
  if (c.dtype == FM_BF16) go(uint16_t{});
  else go(uint32_t{});
  return hipGetLastError();
}

}  // namespace fm
