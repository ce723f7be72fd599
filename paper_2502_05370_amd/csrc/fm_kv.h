// The paged key-value cache: layout of its pages and the arguments its kernels
// share (fm_kv.hip, fm_attn.hip).
#pragma once

#include "fm_internal.h"

namespace fm {

constexpr int kBlockTokens = 16;     // tokens of a block
constexpr int kPieceBytes = 1024;    // 64 bytes of each of its rows
constexpr int kRowPiece = 64;        // bytes of a row in a piece
constexpr int kMaxHeadDim = 256;

// A cache as the kernels take it.  rows of a head are `pieces` x 64 bytes.
struct KvArgs {
  char* pages;
  int32_t* table;
  int32_t* length;
  int32_t* refs;
  int32_t n_slots, max_pages, n_pages, page, layers, heads, head_dim, pieces;
  int64_t page_bytes;

  __device__ __forceinline__ int32_t capacity() const { return max_pages * page; }
  __device__ __forceinline__ int32_t tokens(int32_t len) const {   // a length as it is taken
    return len < 0 ? 0 : (len < capacity() ? len : capacity());
  }
  __device__ __forceinline__ int32_t pages_of(int32_t len) const { return (len + page - 1) / page; }
  __device__ __forceinline__ bool valid(int32_t p) const {
    return static_cast<uint32_t>(p) < static_cast<uint32_t>(n_pages);
  }
  // bytes from a page's start to the keys (kv = 0) or values (1) of a head
  __device__ __forceinline__ int64_t head_offset(int layer, int kv, int head) const {
    return (static_cast<int64_t>(layer * 2 + kv) * heads + head) * (static_cast<int64_t>(page) * pieces * kRowPiece);
  }
};

inline int kv_pieces(int32_t head_dim, int dt) {
  const int bytes = head_dim * (dt == FM_BF16 ? 2 : 4);
  return (bytes + kRowPiece - 1) / kRowPiece;
}
inline int64_t kv_page_bytes(int32_t layers, int32_t heads, int32_t head_dim, int32_t page, int dt) {
  return static_cast<int64_t>(layers) * 2 * heads * page * kv_pieces(head_dim, dt) * kRowPiece;
}
inline KvArgs kv_args(const fm_kv_cache& c) {
  return KvArgs{static_cast<char*>(c.pages), c.table,  c.length, c.refs,     c.n_slots,
                c.max_pages,                 c.n_pages, c.page,  c.layers,   c.heads,
                c.head_dim,                  kv_pieces(c.head_dim, c.dtype),
                kv_page_bytes(c.layers, c.heads, c.head_dim, c.page, c.dtype)};
}

size_t kv_scratch_bytes(const fm_kv_cache& c);
hipError_t launch_kv_resize(const fm_kv_cache& c, const int32_t* delta, uint8_t* granted, uint32_t* flags,
                            void* scratch, hipStream_t st);
hipError_t launch_kv_fork(const fm_kv_cache& c, const int32_t* parent, uint32_t* flags, void* scratch, hipStream_t st);
hipError_t launch_kv_compact(const fm_kv_cache& c, int32_t* live, uint32_t* flags, void* scratch, hipStream_t st);
hipError_t launch_kv_copy(const fm_kv_cache& c, const int32_t* src, const int32_t* dst, int32_t n, uint32_t* flags,
                          void* scratch, hipStream_t st);
// Rows of new tokens; the kernels write k and v only where `read`.
struct KvRows {
  void* k;
  void* v;
  int64_t k_stride, v_stride;   // elements
  const int32_t* offsets;       // [n_slots + 1] or null
  int32_t T, layer;
  const uint8_t* active;        // [n_slots] or null
  uint32_t* flags;
};
hipError_t launch_kv_rows(const fm_kv_cache& c, const KvRows& r, bool read, hipStream_t st);

struct AttnArgs {
  KvArgs c;
  const char* q;
  int64_t q_row;           // bytes
  int32_t q_heads, group;  // query heads, and those per key head
  int32_t layer, window;
  float scale2;            // scale times log2(e)
  uint64_t per_page_inv;   // 2^32 over the blocks of a page, rounded up: exact for up to 2^26 blocks
  const int32_t* first;    // [n_slots] or null
  const uint8_t* active;   // [n_slots] or null
  char* out;
  float* lse;              // [n_slots][q_heads] or null
  uint32_t* flags;
};
bool attn_fits(const fm_kv_cache& c, int32_t q_heads);   // whether its sizes can be handled
size_t attn_workspace_bytes(const fm_kv_cache& c, int32_t q_heads);
hipError_t launch_attn(const AttnArgs& a, fm_dtype dt, void* workspace, hipStream_t st);

}  // namespace fm
