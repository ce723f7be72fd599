// C ABI of the model operators: argument validation and dispatch.  Every entry
// point validates all of its arguments before enqueueing anything; work goes to
// the current device.
#include <hip/hip_runtime.h>

#include "fm_internal.h"

namespace {

using fm::fail;
using fm::hip_fail;
using fm::ok;

// Bounds that keep every grid below 2^32 threads and every position an int32.
constexpr int32_t kMaxWidth = 16384;         // d
constexpr int32_t kMaxFfn = 65536;           // f
constexpr int32_t kMaxTokens = 1 << 24;
constexpr int32_t kMaxRequests = 65536;
constexpr int32_t kMaxGradRows = 1 << 24;
constexpr size_t kMaxSlotBytes = 0xF0000000u;   // a slot is addressed with 32-bit byte offsets

size_t elem(int dt) { return dt == FM_BF16 ? 2 : 4; }

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

fm_status check_rows(const void* table, const char* name, int32_t V, int32_t d, int dt, const int32_t* tokens,
                     int32_t T) {
  if (!fm::valid_dtype(dt)) return fail(FM_ERR_INVALID, "dtype %d is not FM_F32 or FM_BF16", dt);
  if (V < 1) return fail(FM_ERR_INVALID, "V=%d rows: at least 1", V);
  if (d < 1 || d > kMaxWidth) return fail(FM_ERR_INVALID, "d=%d outside [1, %d]", d, kMaxWidth);
  if (T < 0 || T > kMaxTokens) return fail(FM_ERR_INVALID, "T=%d outside [0, %d]", T, kMaxTokens);
  if (T > 0 && (table == nullptr || tokens == nullptr))
    return fail(FM_ERR_INVALID, "%s and tokens must be non-NULL", name);
  if (!aligned(table, elem(dt)) || !aligned(tokens, 4))
    return fail(FM_ERR_INVALID, "%s and tokens must be aligned to their elements", name);
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

// Sizes that fm_moe_experts takes (E and slots aside).
fm_status check_moe_sizes(int32_t d, int32_t f, int dt, int32_t K) {
  if (!fm::valid_dtype(dt)) return fail(FM_ERR_INVALID, "dtype %d is not FM_F32 or FM_BF16", dt);
  if (d < 1 || f < 1) return fail(FM_ERR_INVALID, "d=%d f=%d out of range", d, f);
  if (d % 8 != 0 || f % 8 != 0) return fail(FM_ERR_UNSUPPORTED, "d=%d and f=%d must be multiples of 8", d, f);
  if (d > kMaxWidth || f > kMaxFfn)
    return fail(FM_ERR_UNSUPPORTED, "d=%d beyond %d or f=%d beyond %d", d, kMaxWidth, f, kMaxFfn);
  if (static_cast<size_t>(3) * d * f * elem(dt) > kMaxSlotBytes)
    return fail(FM_ERR_UNSUPPORTED, "d=%d f=%d: one expert's weights exceed %zu bytes", d, f, kMaxSlotBytes);
  if (K < 1 || K > fm::kMaxK) return fail(FM_ERR_INVALID, "K=%d outside [1, %d]", K, fm::kMaxK);
  return FM_OK;
}

}  // namespace

extern "C" {

fm_status fm_embed_lookup(const void* table, int32_t V, int32_t d, fm_dtype dtype, const int32_t* tokens, int32_t T,
                          float scale, void* out, uint32_t* flags, void* stream) {
  if (fm_status st = check_rows(table, "table", V, d, dtype, tokens, T)) return st;
  if (fm_status st = check_flags(flags)) return st;
  if (T == 0) return ok();
  if (out == nullptr || !aligned(out, elem(dtype)))
    return fail(FM_ERR_INVALID, "out must be non-NULL and aligned to its elements");
  const hipError_t e =
      fm::launch_embed_lookup(table, V, d, dtype, tokens, T, scale, out, flags, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "embedding lookup launch");
}

fm_status fm_embed_pool(const void* table, int32_t V, int32_t d, fm_dtype dtype, const int32_t* tokens, int32_t T,
                        const int32_t* offsets, int32_t B, float scale, void* out, uint32_t* flags, void* stream) {
  if (fm_status st = check_rows(table, "table", V, d, dtype, tokens, T)) return st;
  if (fm_status st = check_flags(flags)) return st;
  if (B < 0 || B > kMaxRequests) return fail(FM_ERR_INVALID, "B=%d outside [0, %d]", B, kMaxRequests);
  if (B == 0) return ok();
  if (offsets == nullptr || out == nullptr || !aligned(offsets, 4) || !aligned(out, 2))
    return fail(FM_ERR_INVALID, "offsets and out must be non-NULL and aligned to their elements");
  const hipError_t e = fm::launch_embed_pool(table, V, d, dtype, tokens, T, offsets, B, scale,
                                             static_cast<uint16_t*>(out), flags, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "embedding pool launch");
}

size_t fm_embed_grad_scratch_bytes(int32_t T_max, int32_t V) {
  if (T_max < 0 || T_max > kMaxTokens || V < 1 || V > kMaxGradRows) return 0;
  return fm::embed_grad_scratch_bytes(T_max, V);
}

fm_status fm_embed_grad(const void* dout, fm_dtype dtype, const int32_t* tokens, int32_t T, int32_t V, int32_t d,
                        float scale, int32_t accumulate, void* dtable, fm_dtype grad_dtype, void* scratch,
                        size_t scratch_bytes, uint32_t* flags, void* stream) {
  if (fm_status st = check_rows(dout, "dout", V, d, dtype, tokens, T)) return st;
  if (fm_status st = check_flags(flags)) return st;
  if (V > kMaxGradRows) return fail(FM_ERR_UNSUPPORTED, "V=%d beyond %d", V, kMaxGradRows);
  if (!fm::valid_dtype(grad_dtype)) return fail(FM_ERR_INVALID, "grad_dtype %d is not FM_F32 or FM_BF16", grad_dtype);
  if (dtable == nullptr || !aligned(dtable, elem(grad_dtype)))
    return fail(FM_ERR_INVALID, "dtable must be non-NULL and aligned to its elements");
  if (fm_status st = check_buffer(scratch, scratch_bytes, fm::embed_grad_scratch_bytes(T, V), "scratch")) return st;
  const hipError_t e = fm::launch_embed_grad(dout, dtype, tokens, T, V, d, scale, accumulate != 0, dtable, grad_dtype,
                                             scratch, flags, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "embedding gradient launch");
}

fm_status fm_moe_route(const void* x, const void* gate, fm_dtype dtype, int32_t T, int32_t d, int32_t E, int32_t K,
                       int32_t renorm, const uint8_t* active, void* probs_out, fm_dtype probs_dtype,
                       int64_t probs_stride, int32_t* ids_out, float* weight_out, uint64_t* mask_out, void* stream) {
  if (!fm::valid_dtype(dtype)) return fail(FM_ERR_INVALID, "dtype %d is not FM_F32 or FM_BF16", dtype);
  if (!fm::valid_dtype(probs_dtype))
    return fail(FM_ERR_INVALID, "probs_dtype %d is not FM_F32 or FM_BF16", probs_dtype);
  if (T < 0 || T > kMaxTokens) return fail(FM_ERR_INVALID, "T=%d outside [0, %d]", T, kMaxTokens);
  if (E < 1) return fail(FM_ERR_INVALID, "E=%d experts: at least 1", E);
  if (E > fm::kMaxE) return fail(FM_ERR_UNSUPPORTED, "E=%d exceeds %d experts per layer", E, fm::kMaxE);
  if (K < 1 || K > fm::kMaxK || K > E) return fail(FM_ERR_INVALID, "K=%d outside [1, min(%d, E=%d)]", K, fm::kMaxK, E);
  if (d < 1) return fail(FM_ERR_INVALID, "d=%d: at least 1", d);
  if (d % 8 != 0) return fail(FM_ERR_UNSUPPORTED, "d=%d is not a multiple of 8", d);
  if (d > kMaxWidth) return fail(FM_ERR_UNSUPPORTED, "d=%d beyond %d", d, kMaxWidth);
  if (probs_stride < E) return fail(FM_ERR_INVALID, "probs_stride=%lld is below E=%d", static_cast<long long>(probs_stride), E);
  if (T == 0) return ok();
  if (x == nullptr || gate == nullptr || probs_out == nullptr || ids_out == nullptr || weight_out == nullptr)
    return fail(FM_ERR_INVALID, "x, gate, probs_out, ids_out and weight_out must be non-NULL");
  if (!aligned(x, 16) || !aligned(gate, 16)) return fail(FM_ERR_INVALID, "x and gate must be 16-byte aligned");
  if (!aligned(probs_out, elem(probs_dtype)) || !aligned(ids_out, 4) || !aligned(weight_out, 4) || !aligned(mask_out, 8))
    return fail(FM_ERR_INVALID, "outputs must be aligned to their elements");
  const fm::RouteArgs a{x,      gate,         T,       d,          E,        K, renorm != 0, active,
                        probs_out, probs_stride, ids_out, weight_out, mask_out};
  const hipError_t e = fm::launch_moe_route(a, dtype, probs_dtype, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "gate launch");
}

size_t fm_moe_workspace_bytes(int32_t d, int32_t f, fm_dtype dtype, int32_t T_max, int32_t K) {
  if (check_moe_sizes(d, f, dtype, K) != FM_OK || T_max < 1 || T_max > kMaxTokens) return 0;
  return fm::moe_workspace_bytes(d, f, dtype, T_max, K);
}

fm_status fm_moe_experts(const fm_expert_cache* c, const void* x, const int32_t* ids, const float* weight, int32_t T,
                         int32_t K, const void* residual, void* out, uint32_t* flags, void* workspace,
                         size_t workspace_bytes, void* stream) {
  if (c == nullptr) return fail(FM_ERR_INVALID, "expert cache is NULL");
  if (fm_status st = check_moe_sizes(c->d, c->f, c->dtype, K)) return st;
  if (c->E < 1 || c->n_slots < 1) return fail(FM_ERR_INVALID, "E=%d n_slots=%d: at least 1", c->E, c->n_slots);
  if (c->E > fm::kMaxE) return fail(FM_ERR_UNSUPPORTED, "E=%d exceeds %d experts per layer", c->E, fm::kMaxE);
  if (T < 0 || T > kMaxTokens) return fail(FM_ERR_INVALID, "T=%d outside [0, %d]", T, kMaxTokens);
  if (fm_status st = check_flags(flags)) return st;
  if (T == 0) return ok();
  if (c->slots == nullptr || c->slot_of == nullptr) return fail(FM_ERR_INVALID, "slots and slot_of must be non-NULL");
  if (x == nullptr || ids == nullptr || weight == nullptr || out == nullptr)
    return fail(FM_ERR_INVALID, "x, ids, weight and out must be non-NULL");
  if (!aligned(c->slots, 16) || !aligned(x, 16) || !aligned(residual, 16) || !aligned(out, 16))
    return fail(FM_ERR_INVALID, "slots, x, residual and out must be 16-byte aligned");
  if (!aligned(c->slot_of, 4) || !aligned(ids, 4) || !aligned(weight, 4))
    return fail(FM_ERR_INVALID, "slot_of, ids and weight must be 4-byte aligned");
  const size_t need = fm::moe_workspace_bytes(c->d, c->f, c->dtype, T, K);
  if (fm_status st = check_buffer(workspace, workspace_bytes, need, "workspace")) return st;
  const hipError_t e = fm::launch_moe_experts(*c, x, ids, weight, T, K, residual, out, flags, workspace,
                                              static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "experts launch");
}

}  // extern "C"
