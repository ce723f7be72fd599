// The gate of an MoE layer: logits x[t] . gate[e], their softmax over the
// layer's experts and the K largest.  The probabilities are a row of an expert
// map (Section 4.1) or of a trajectory query (Section 4.2.2) and are written
// there.
//
// A batch of decode tokens is bound by latency (one workgroup reads E d values,
// 246 KB for 60 experts of 2,048: 11 us, 5 of them without the gate), a prefill by
// reading x (8,192 x 4,096 bf16, 16 experts: 18 us, 3.8 TB/s of x and the gate's
// 64 MB from the L2).  A workgroup takes 16 tokens per tile; its wavefronts split d, so that the loads of a decode call are
// in flight at once (of rows of up to 4 KB; longer ones take another turn per 4 KB),
// and join their sums in LDS in a fixed order.  One workgroup thus reads the whole
// gate for up to 16 tokens: the time grows with E d (64 experts of 8,192: 28 us).  One
// wavefront then holds one token's logits, an expert per lane.
#include "fm_internal.h"
#include "fm_mma.h"

namespace fm {

namespace {

// Larger float -> larger key; -0 as +0; NaN lowest.
__device__ __forceinline__ uint32_t logit_key(float l) {
  if (l != l) return 0u;
  const uint32_t u = __float_as_uint(l + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

template <typename T, int TT, int NE, int NW, int PD>
__global__ void __launch_bounds__(NW * kWave) k_route(RouteArgs a, bool probs_bf16) {
  constexpr int kLd = NE * 16 + 1;   // (an odd row length keeps the tile's rows apart)
  __shared__ float red[NW][16 * TT][kLd];
  const int lane = threadIdx.x % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c = lane % 16;
  const int g = lane / 16;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * (16 * TT);
  const int n_tok = a.T - t0 < 16 * TT ? static_cast<int>(a.T - t0) : 16 * TT;
  const uint32_t rb = static_cast<uint32_t>(a.d) * sizeof(T);
  // rows past the batch and past the experts lie past the buffers' ends
  const __amdgpu_buffer_rsrc_t rs_x =
      row_buffer(static_cast<const char*>(a.x) + t0 * rb, static_cast<uint32_t>(n_tok) * rb);
  const __amdgpu_buffer_rsrc_t rs_g = row_buffer(a.gate, static_cast<uint32_t>(a.E) * rb);
  // which of this workgroup's tokens have a request, a token per lane (loaded
  // now, looked at after the products)
  uint32_t live = 1;
  if (a.active != nullptr && lane < n_tok) live = a.active[t0 + lane];
  floatx4 acc[TT][NE];
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int j = 0; j < NE; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

  RowPairs tokens[TT], experts[NE];
#pragma unroll
  for (int i = 0; i < TT; ++i) tokens[i] = RowPairs(16 * i, n_tok, rb, 0u);
#pragma unroll
  for (int j = 0; j < NE; ++j) experts[j] = RowPairs(16 * j, a.E, rb, 0u);
  uint32x4 fx[PD][TT][2], fg[PD][NE][2];
  auto load = [&](int p, uint32_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TT; ++i) tokens[i].template load<kStream>(rs_x, k, rb, fx[p][i]);
#pragma unroll
    for (int j = 0; j < NE; ++j) experts[j].template load<kKeep>(rs_g, k, rb, fg[p][j]);
  };
  // the wavefronts deal the rows' lines among themselves
  constexpr uint32_t kStride = NW * RowPairs::kBytes;
  const uint32_t k0 = static_cast<uint32_t>(wv) * RowPairs::kBytes;
#pragma unroll
  for (int p = 0; p < PD; ++p) load(p, k0 + p * kStride);
  for (uint32_t k = k0; k < rb; k += PD * kStride) {
#pragma unroll
    for (int p = 0; p < PD; ++p) {
      uint32x4 sx[TT][2];
#pragma unroll
      for (int i = 0; i < TT; ++i) RowPairs::steps(fx[p][i], sx[i]);
#pragma unroll
      for (int j = 0; j < NE; ++j) {
        uint32x4 sg[2];
        RowPairs::steps(fg[p][j], sg);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < TT; ++i) acc[i][j] = mma_step<T>(sx[i][s], sg[s], acc[i][j]);
      }
      load(p, k + (p + PD) * kStride);
    }
  }
  // lane 16 g + c of a tile holds tokens 4 g .. 4 g + 3 of expert c
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int j = 0; j < NE; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) red[wv][16 * i + 4 * g + r][16 * j + c] = acc[i][j][r];
  __syncthreads();
  const uint64_t on_mask = __ballot(live != 0);

  for (int i = wv; i < n_tok; i += NW) {
    const int64_t t = t0 + i;
    const bool expert = lane < a.E;
    float l = 0.0f;
    if (lane < NE * 16) {
#pragma unroll
      for (int w = 0; w < NW; ++w) l += red[w][i][lane];
    }
    const bool on = (on_mask >> i) & 1ull;
    float top = expert ? l : -__builtin_inff();
#pragma unroll
    for (int m = kWave / 2; m >= 1; m >>= 1) top = fmaxf(top, __shfl_xor(top, m, kWave));
    const float e = expert ? expf(l - top) : 0.0f;
    float sum = e;
#pragma unroll
    for (int m = kWave / 2; m >= 1; m >>= 1) sum += __shfl_xor(sum, m, kWave);
    const float p = e / sum;
    // place in the order by logit: the experts before this one (an equal logit
    // comes before where its index is lower; keys stay below 2^32 - 1)
    const uint32_t key = expert ? logit_key(l) : 0u;
    int rank = expert ? 0 : kMaxE;
#pragma unroll
    for (int j = 0; j < NE * 16; ++j) {
      const uint32_t o = __builtin_amdgcn_readlane(key, j) + (j < lane ? 1u : 0u);
      rank += o > key && j < a.E ? 1 : 0;
    }
    const bool chosen = rank < a.K;
    float w = chosen ? p : 0.0f;
    if (a.renorm) {
      float kept = w;
#pragma unroll
      for (int m = kWave / 2; m >= 1; m >>= 1) kept += __shfl_xor(kept, m, kWave);
      w = w / kept;
    }
    const uint64_t mask = __ballot(chosen);
    if (expert) {
      const float v = on ? p : 0.0f;
      if (probs_bf16)
        static_cast<__bf16*>(a.probs)[t * a.probs_stride + lane] = static_cast<__bf16>(v);
      else
        static_cast<float*>(a.probs)[t * a.probs_stride + lane] = v;
    }
    if (chosen) {
      a.ids[t * a.K + rank] = on ? lane : -1;
      a.weight[t * a.K + rank] = on ? w : 0.0f;
    }
    if (lane == 0 && a.mask != nullptr) a.mask[t] = on ? mask : 0ull;
  }
}

template <typename T, int NE>
void route(const RouteArgs& a, bool probs_bf16, hipStream_t st) {
  // Few tokens: 16 wavefronts on 16 tokens, 4 KB of every row in flight.  Many:
  // eight wavefronts, two workgroups per CU, on 16 tokens each, or 32 where the
  // gate's tiles outweigh the tokens' (its lines come from the L2 once per
  // workgroup).  Us of the first and the second form at 2,048 and 8,192 tokens,
  // bf16: E 16 d 4,096 9.9 and 10.1, 20.1 and 18.6; E 60 d 2,048 14.7 and 20.0, 30.0
  // and 22.0; E 32 d 1,024 8.4 and 7.5, 15.1 and 10.9; float32 E 60 d 2,048 21.9 and
  // 35.6, 43.1 and 39.6.  The first takes a second turn of workgroups only from
  // 4,097 tokens on and is ahead until then at E 60 (4,096 tokens: 16.2 and 21.4),
  // while at E 16 they are within 6%.
  constexpr int TT = NE == 4 ? 2 : 1;
  if (a.T <= 2048) {
    k_route<T, 1, NE, 16, 2><<<static_cast<unsigned>((a.T + 15) / 16), 16 * kWave, 0, st>>>(a, probs_bf16);
  } else {
    const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(a.T) + 16 * TT - 1) / (16 * TT));
    k_route<T, TT, NE, 8, NE == 1 ? 4 : 2><<<grid, 8 * kWave, 0, st>>>(a, probs_bf16);
  }
}

}  // namespace

hipError_t launch_moe_route(const RouteArgs& a, fm_dtype dt, fm_dtype probs_dt, hipStream_t st) {
  const bool pb = probs_dt == FM_BF16;
  const int ne = (a.E + 15) / 16;
  if (dt == FM_BF16) {
    if (ne == 1) route<uint16_t, 1>(a, pb, st);
    else if (ne == 2) route<uint16_t, 2>(a, pb, st);
    else route<uint16_t, 4>(a, pb, st);
  } else {
    if (ne == 1) route<float, 1>(a, pb, st);
    else if (ne == 2) route<float, 2>(a, pb, st);
    else route<float, 4>(a, pb, st);
  }
  return hipGetLastError();
}

}  // namespace fm
