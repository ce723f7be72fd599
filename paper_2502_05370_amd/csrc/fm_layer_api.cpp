// C ABI of the paged cache, the attention over it and the norms around a block:
// argument validation and dispatch.  Every entry point validates all of its
// arguments before enqueueing anything; work goes to the current device.
#include <hip/hip_runtime.h>

#include <cmath>

#include "fm_kv.h"
#include "fm_norm.h"

namespace {

using fm::fail;
using fm::hip_fail;
using fm::ok;

constexpr int32_t kMaxSlots = 65536;
constexpr int32_t kMaxPages = 1 << 24;
constexpr int64_t kMaxEntries = int64_t{1} << 28;
constexpr int64_t kMaxCapacity = int64_t{1} << 30;   // tokens of a slot: places are int32 and pages' reciprocals exact
constexpr int64_t kMaxPageBytes = int64_t{1} << 31;
constexpr int32_t kMaxTokens = 1 << 24;
constexpr int32_t kMaxWidth = 16384;
constexpr int64_t kMaxStride = int64_t{1} << 40;

size_t elem(int dt) { return dt == FM_BF16 ? 2 : 4; }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

fm_status check_page(int32_t layers, int32_t heads, int32_t head_dim, int32_t page, int dt) {
  if (!fm::valid_dtype(dt)) return fail(FM_ERR_INVALID, "dtype %d is not FM_F32 or FM_BF16", dt);
  if (layers < 1 || layers > 1024) return fail(FM_ERR_INVALID, "layers=%d outside [1, 1024]", layers);
  if (heads < 1 || heads > 1024) return fail(FM_ERR_INVALID, "heads=%d outside [1, 1024]", heads);
  if (head_dim < 1 || page < 1) return fail(FM_ERR_INVALID, "head_dim=%d page=%d: at least 1", head_dim, page);
  if (head_dim % 8 != 0 || head_dim > fm::kMaxHeadDim)
    return fail(FM_ERR_UNSUPPORTED, "head_dim=%d is not a multiple of 8 up to %d", head_dim, fm::kMaxHeadDim);
  if (page % 16 != 0 || page > 1024) return fail(FM_ERR_UNSUPPORTED, "page=%d is not a multiple of 16 up to 1024", page);
  if (fm::kv_page_bytes(layers, heads, head_dim, page, dt) > kMaxPageBytes)
    return fail(FM_ERR_UNSUPPORTED, "a page of %d tokens exceeds %lld bytes", page,
                static_cast<long long>(kMaxPageBytes));
  return FM_OK;
}

fm_status check_sizes(const fm_kv_cache* c) {
  if (c == nullptr) return fail(FM_ERR_INVALID, "cache is NULL");
  if (fm_status st = check_page(c->layers, c->heads, c->head_dim, c->page, c->dtype)) return st;
  if (c->n_slots < 1 || c->n_slots > kMaxSlots)
    return fail(FM_ERR_INVALID, "n_slots=%d outside [1, %d]", c->n_slots, kMaxSlots);
  if (c->n_pages < 1 || c->n_pages > kMaxPages)
    return fail(FM_ERR_INVALID, "n_pages=%d outside [1, %d]", c->n_pages, kMaxPages);
  if (c->max_pages < 1) return fail(FM_ERR_INVALID, "max_pages=%d: at least 1", c->max_pages);
  if (static_cast<int64_t>(c->max_pages) * c->page > kMaxCapacity ||
      static_cast<int64_t>(c->max_pages) * c->n_slots > kMaxEntries)
    return fail(FM_ERR_UNSUPPORTED, "max_pages=%d: a slot's tokens or the table exceed their limits", c->max_pages);
  return FM_OK;
}

fm_status check_cache(const fm_kv_cache* c) {
  if (fm_status st = check_sizes(c)) return st;
  if (c->pages == nullptr || c->table == nullptr || c->length == nullptr || c->refs == nullptr)
    return fail(FM_ERR_INVALID, "pages, table, length and refs must be non-NULL");
  if (!aligned(c->pages, fm::kAlign)) return fail(FM_ERR_INVALID, "pages must be %zu-byte aligned", fm::kAlign);
  if (!aligned(c->table, 4) || !aligned(c->length, 4) || !aligned(c->refs, 4))
    return fail(FM_ERR_INVALID, "table, length and refs must be 4-byte aligned");
  return FM_OK;
}

fm_status check_flags(const uint32_t* flags) {
  if (!aligned(flags, 4)) return fail(FM_ERR_INVALID, "flags must be 4-byte aligned");
  return FM_OK;
}

fm_status check_buffer(const void* p, size_t bytes, size_t need, const char* name) {
  if (p == nullptr) return fail(FM_ERR_INVALID, "%s is NULL", name);
  if (!aligned(p, fm::kAlign)) return fail(FM_ERR_INVALID, "%s must be %zu-byte aligned", name, fm::kAlign);
  if (bytes < need)
    return fail(FM_ERR_INVALID, "%s of %zu bytes is smaller than the %zu bytes required", name, bytes, need);
  return FM_OK;
}

fm_status check_layer(const fm_kv_cache* c, int32_t layer) {
  if (layer < 0 || layer >= c->layers) return fail(FM_ERR_INVALID, "layer=%d outside [0, %d)", layer, c->layers);
  return FM_OK;
}

// Rows of `width` elements at a stride.
fm_status check_rows(const void* p, int64_t stride, int64_t width, int dt, const char* name) {
  if (p == nullptr) return fail(FM_ERR_INVALID, "%s is NULL", name);
  if (!aligned(p, 16)) return fail(FM_ERR_INVALID, "%s must be 16-byte aligned", name);
  if (stride < width || stride > kMaxStride)
    return fail(FM_ERR_INVALID, "%s_stride=%lld is below %lld", name, static_cast<long long>(stride),
                static_cast<long long>(width));
  if (stride * static_cast<int64_t>(elem(dt)) % 16 != 0)
    return fail(FM_ERR_INVALID, "%s_stride=%lld is not a multiple of 16 bytes", name, static_cast<long long>(stride));
  return FM_OK;
}

fm_status rows_call(const fm_kv_cache* c, int32_t layer, void* k, int64_t k_stride, void* v, int64_t v_stride,
                    const int32_t* offsets, int32_t T, const uint8_t* active, uint32_t* flags, void* stream, bool read) {
  if (fm_status st = check_cache(c)) return st;
  if (fm_status st = check_layer(c, layer)) return st;
  if (fm_status st = check_flags(flags)) return st;
  if (T < 0 || T > kMaxTokens) return fail(FM_ERR_INVALID, "T=%d outside [0, %d]", T, kMaxTokens);
  if (offsets == nullptr && T != c->n_slots)
    return fail(FM_ERR_INVALID, "T=%d rows for %d slots without offsets", T, c->n_slots);
  if (!aligned(offsets, 4)) return fail(FM_ERR_INVALID, "offsets must be 4-byte aligned");
  if (T == 0) return ok();
  const int64_t width = static_cast<int64_t>(c->heads) * c->head_dim;
  if (fm_status st = check_rows(k, k_stride, width, c->dtype, "k")) return st;
  if (fm_status st = check_rows(v, v_stride, width, c->dtype, "v")) return st;
  if (read && k == v) return fail(FM_ERR_INVALID, "k and v must not be the same");
  const fm::KvRows r{k, v, k_stride, v_stride, offsets, T, layer, active, flags};
  const hipError_t e = fm::launch_kv_rows(*c, r, read, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, read ? "cache read launch" : "cache write launch");
}

fm_status check_attn(const fm_kv_cache* c, int32_t q_heads) {
  if (q_heads < 1 || q_heads > 1024) return fail(FM_ERR_INVALID, "q_heads=%d outside [1, 1024]", q_heads);
  if (q_heads % c->heads != 0)
    return fail(FM_ERR_INVALID, "q_heads=%d is not a multiple of heads=%d", q_heads, c->heads);
  if (!fm::attn_fits(*c, q_heads))
    return fail(FM_ERR_UNSUPPORTED, "n_slots=%d of %d pages, q_heads=%d: more work than 2^37 blocks", c->n_slots,
                c->max_pages, q_heads);
  return FM_OK;
}

// The arguments that the norm and its gradient share.
fm_status check_norm(const void* x, const void* y, const void* post, const void* gate, int kind, const void* pre,
                     float scale, float eps, int32_t T, int32_t d, int dt) {
  if (!fm::valid_dtype(dt)) return fail(FM_ERR_INVALID, "dtype %d is not FM_F32 or FM_BF16", dt);
  if (T < 0 || T > kMaxTokens) return fail(FM_ERR_INVALID, "T=%d outside [0, %d]", T, kMaxTokens);
  if (d < 1) return fail(FM_ERR_INVALID, "d=%d: at least 1", d);
  if (d % 8 != 0) return fail(FM_ERR_UNSUPPORTED, "d=%d is not a multiple of 8", d);
  if (d > kMaxWidth) return fail(FM_ERR_UNSUPPORTED, "d=%d beyond %d", d, kMaxWidth);
  if (kind < FM_GATE_NONE || kind > FM_GATE_EACH) return fail(FM_ERR_INVALID, "gate kind %d is not one of 0 to 3", kind);
  if (!(eps >= 0.0f) || std::isinf(eps)) return fail(FM_ERR_INVALID, "eps=%g must be finite and at least 0", eps);
  if ((gate == nullptr) != (kind == FM_GATE_NONE) && T > 0)
    return fail(FM_ERR_INVALID, "gate must be given exactly where its kind is not FM_GATE_NONE");
  if (T > 0 && x == nullptr) return fail(FM_ERR_INVALID, "x is NULL");
  if (T > 0 && y == nullptr && (post != nullptr || kind != FM_GATE_NONE))
    return fail(FM_ERR_INVALID, "post and gate need y");
  if (!aligned(x, 16) || !aligned(y, 16) || !aligned(post, 16) || !aligned(pre, 16) ||
      !aligned(gate, kind == FM_GATE_TOKEN ? elem(dt) : 16))
    return fail(FM_ERR_INVALID, "x, y, post, pre and gate must be 16-byte aligned (a gate per token to its elements)");
  return FM_OK;
}

}  // namespace

extern "C" {

size_t fm_kv_page_bytes(int32_t layers, int32_t heads, int32_t head_dim, int32_t page, fm_dtype dtype) {
  if (check_page(layers, heads, head_dim, page, dtype) != FM_OK) return 0;
  return static_cast<size_t>(fm::kv_page_bytes(layers, heads, head_dim, page, dtype));
}

size_t fm_kv_scratch_bytes(const fm_kv_cache* c) {
  if (check_sizes(c) != FM_OK) return 0;
  return fm::kv_scratch_bytes(*c);
}

fm_status fm_kv_resize(const fm_kv_cache* c, const int32_t* delta, uint8_t* granted_out, uint32_t* flags,
                       void* scratch, size_t scratch_bytes, void* stream) {
  if (fm_status st = check_cache(c)) return st;
  if (fm_status st = check_flags(flags)) return st;
  if (delta == nullptr || !aligned(delta, 4)) return fail(FM_ERR_INVALID, "delta must be non-NULL and 4-byte aligned");
  if (fm_status st = check_buffer(scratch, scratch_bytes, fm::kv_scratch_bytes(*c), "scratch")) return st;
  const hipError_t e = fm::launch_kv_resize(*c, delta, granted_out, flags, scratch, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "cache resize launch");
}

fm_status fm_kv_fork(const fm_kv_cache* c, const int32_t* parent, uint32_t* flags, void* scratch,
                     size_t scratch_bytes, void* stream) {
  if (fm_status st = check_cache(c)) return st;
  if (fm_status st = check_flags(flags)) return st;
  if (parent == nullptr || !aligned(parent, 4))
    return fail(FM_ERR_INVALID, "parent must be non-NULL and 4-byte aligned");
  if (fm_status st = check_buffer(scratch, scratch_bytes, fm::kv_scratch_bytes(*c), "scratch")) return st;
  const hipError_t e = fm::launch_kv_fork(*c, parent, flags, scratch, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "cache fork launch");
}

fm_status fm_kv_compact(const fm_kv_cache* c, int32_t* live_out, uint32_t* flags, void* scratch,
                        size_t scratch_bytes, void* stream) {
  if (fm_status st = check_cache(c)) return st;
  if (fm_status st = check_flags(flags)) return st;
  if (!aligned(live_out, 4)) return fail(FM_ERR_INVALID, "live_out must be 4-byte aligned");
  if (fm_status st = check_buffer(scratch, scratch_bytes, fm::kv_scratch_bytes(*c), "scratch")) return st;
  const hipError_t e = fm::launch_kv_compact(*c, live_out, flags, scratch, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "cache compaction launch");
}

fm_status fm_kv_copy(const fm_kv_cache* c, const int32_t* src, const int32_t* dst, int32_t n, uint32_t* flags,
                     void* scratch, size_t scratch_bytes, void* stream) {
  if (fm_status st = check_cache(c)) return st;
  if (fm_status st = check_flags(flags)) return st;
  if (n < 0 || n > c->n_pages) return fail(FM_ERR_INVALID, "n=%d outside [0, n_pages=%d]", n, c->n_pages);
  if (fm_status st = check_buffer(scratch, scratch_bytes, fm::kv_scratch_bytes(*c), "scratch")) return st;
  if (n == 0) return ok();
  if (src == nullptr || dst == nullptr || !aligned(src, 4) || !aligned(dst, 4))
    return fail(FM_ERR_INVALID, "src and dst must be non-NULL and 4-byte aligned");
  const hipError_t e = fm::launch_kv_copy(*c, src, dst, n, flags, scratch, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "cache copy launch");
}

fm_status fm_kv_write(const fm_kv_cache* c, int32_t layer, const void* k, int64_t k_stride, const void* v,
                      int64_t v_stride, const int32_t* offsets, int32_t T, const uint8_t* active, uint32_t* flags,
                      void* stream) {
  return rows_call(c, layer, const_cast<void*>(k), k_stride, const_cast<void*>(v), v_stride, offsets, T, active, flags,
                   stream, false);
}

fm_status fm_kv_read(const fm_kv_cache* c, int32_t layer, void* k, int64_t k_stride, void* v, int64_t v_stride,
                     const int32_t* offsets, int32_t T, const uint8_t* active, uint32_t* flags, void* stream) {
  return rows_call(c, layer, k, k_stride, v, v_stride, offsets, T, active, flags, stream, true);
}

size_t fm_attn_workspace_bytes(const fm_kv_cache* c, int32_t q_heads) {
  if (check_sizes(c) != FM_OK || check_attn(c, q_heads) != FM_OK) return 0;
  return fm::attn_workspace_bytes(*c, q_heads);
}

fm_status fm_attn_decode(const fm_kv_cache* c, int32_t layer, const void* q, int64_t q_stride, int32_t q_heads,
                         float scale, int32_t window, const int32_t* first, const uint8_t* active, void* out,
                         float* lse_out, uint32_t* flags, void* workspace, size_t workspace_bytes, void* stream) {
  if (fm_status st = check_cache(c)) return st;
  if (fm_status st = check_layer(c, layer)) return st;
  if (fm_status st = check_attn(c, q_heads)) return st;
  if (fm_status st = check_flags(flags)) return st;
  if (fm_status st = check_rows(q, q_stride, static_cast<int64_t>(q_heads) * c->head_dim, c->dtype, "q")) return st;
  if (window < 0) return fail(FM_ERR_INVALID, "window=%d: 0 (none) or more", window);
  const float scale2 = scale * 1.44269504088896341f;   // log2(e): weights are powers of two
  if (!std::isfinite(scale2)) return fail(FM_ERR_INVALID, "scale=%g must be finite, with log2(e) times it", scale);
  if (out == nullptr || !aligned(out, 16)) return fail(FM_ERR_INVALID, "out must be non-NULL and 16-byte aligned");
  if (out == q) return fail(FM_ERR_INVALID, "out must not be q");
  if (!aligned(first, 4) || !aligned(lse_out, 4)) return fail(FM_ERR_INVALID, "first and lse_out must be 4-byte aligned");
  if (fm_status st = check_buffer(workspace, workspace_bytes, fm::attn_workspace_bytes(*c, q_heads), "workspace"))
    return st;
  const int32_t group = q_heads / c->heads;
  const uint64_t per_page = static_cast<uint64_t>(c->page / fm::kBlockTokens);
  const fm::AttnArgs a{fm::kv_args(*c),
                       static_cast<const char*>(q),
                       q_stride * static_cast<int64_t>(elem(c->dtype)),
                       q_heads,
                       group,
                       layer,
                       window,
                       scale2,
                       ((uint64_t{1} << 32) + per_page - 1) / per_page,
                       first,
                       active,
                       static_cast<char*>(out),
                       lse_out,
                       flags};
  const hipError_t e = fm::launch_attn(a, c->dtype, workspace, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "attention launch");
}

fm_status fm_block_norm(const void* x, const void* y, const void* post, const void* gate, fm_gate_kind gate_kind,
                        float scale, const void* pre, float eps, int32_t T, int32_t d, fm_dtype dtype, void* r_out,
                        void* h_out, void* stream) {
  if (fm_status st = check_norm(x, y, post, gate, gate_kind, pre, scale, eps, T, d, dtype)) return st;
  if (T == 0) return ok();
  if (y == nullptr && pre == nullptr) return fail(FM_ERR_INVALID, "y or pre must be non-NULL");
  if ((y == nullptr) != (r_out == nullptr)) return fail(FM_ERR_INVALID, "r_out must be given exactly where y is");
  if ((pre == nullptr) != (h_out == nullptr)) return fail(FM_ERR_INVALID, "h_out must be given exactly where pre is");
  if (!aligned(r_out, 16) || !aligned(h_out, 16)) return fail(FM_ERR_INVALID, "outputs must be 16-byte aligned");
  if (r_out == h_out) return fail(FM_ERR_INVALID, "r_out and h_out must not be the same");
  const fm::NormArgs a{x, y, post, gate, pre, gate_kind, scale, eps, T, d, r_out, h_out};
  const hipError_t e = fm::launch_norm(a, dtype, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "norm launch");
}

size_t fm_block_norm_scratch_bytes(int32_t T_max, int32_t d) {
  if (T_max < 0 || T_max > kMaxTokens || d < 8 || d > kMaxWidth || d % 8 != 0) return 0;
  return fm::norm_scratch_bytes(T_max, d);
}

fm_status fm_block_norm_grad(const void* dr, const void* dh, const void* x, const void* y, const void* post,
                             const void* gate, fm_gate_kind gate_kind, float scale, const void* pre, float eps,
                             int32_t T, int32_t d, fm_dtype dtype, int32_t accumulate, void* dx, void* dy,
                             float* dpost, void* dgate, float* dpre, void* scratch, size_t scratch_bytes,
                             void* stream) {
  if (fm_status st = check_norm(x, y, post, gate, gate_kind, pre, scale, eps, T, d, dtype)) return st;
  const bool rows = T > 0;
  if ((dpost == nullptr) != (post == nullptr) || (dpre == nullptr) != (pre == nullptr))
    return fail(FM_ERR_INVALID, "dpost and dpre must be given exactly where post and pre are");
  if ((dgate == nullptr) != (gate_kind == FM_GATE_NONE) && (rows || gate_kind == FM_GATE_CHANNEL))
    return fail(FM_ERR_INVALID, "dgate must be given exactly where gate is");
  if (rows && dr == nullptr && dh == nullptr) return fail(FM_ERR_INVALID, "dr or dh must be non-NULL");
  if (rows && (dh == nullptr) != (pre == nullptr)) return fail(FM_ERR_INVALID, "dh must be given exactly where pre is");
  if (rows && (dx == nullptr || (dy == nullptr) != (y == nullptr)))
    return fail(FM_ERR_INVALID, "dx must be non-NULL, and dy exactly where y is");
  if (!aligned(dr, 16) || !aligned(dh, 16) || !aligned(dx, 16) || !aligned(dy, 16) || !aligned(dpost, 4) ||
      !aligned(dpre, 4) || !aligned(dgate, gate_kind == FM_GATE_EACH ? 16 : 4))
    return fail(FM_ERR_INVALID, "gradients of [T][d] must be 16-byte aligned, the others 4-byte aligned");
  const void* outs[] = {dx, dy, dpost, dgate, dpre};
  for (int i = 0; i < 5; ++i)
    for (int j = 0; j < i; ++j)
      if (outs[i] != nullptr && outs[i] == outs[j]) return fail(FM_ERR_INVALID, "no two gradients may be the same");
  if (fm_status st = check_buffer(scratch, scratch_bytes, fm::norm_scratch_bytes(T, d), "scratch")) return st;
  const fm::NormGradArgs a{{x, y, post, gate, pre, gate_kind, scale, eps, T, d, nullptr, nullptr},
                           dr, dh, accumulate, dx, dy, dpost, dgate, dpre, static_cast<float*>(scratch)};
  const hipError_t e = fm::launch_norm_grad(a, dtype, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "norm gradient launch");
}

}  // extern "C"
