// Norms after and before a block, with the block's gate and scale on its way into
// the residual stream, and their gradient.
//
// A row passes through registers once: W wavefronts hold it, V vectors of 16 bytes
// per thread.  Forward: the sum of y^2, then that of r^2.  Gradient (g gate, s
// scale, ^ a normed row):
//   dz = dh pre            dr' = dr + (dz - r^ mean(dz r^)) / |r|      = dx
//   dn = s dr' g           dgate = s dr' n
//   dz' = dn post          dy = (dz' - y^ mean(dz' y^)) / |y|
//   dpre = sum over rows of dh r^,  dpost = sum of dn y^
// with r and n made again from x and y, which costs one more sum over the row and
// reads no more than the stored r would.  Memory bounds both.
#include "fm_device.h"
#include "fm_norm.h"

namespace fm {

namespace {

template <int CTRL>
__device__ __forceinline__ float ror(float v) {   // lanes of a row of 16 turned
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// Sum over the wavefront, the same bits in every lane.
__device__ __forceinline__ float wave_sum(float v) {
  v += ror<0x128>(v);   // by 8, 4, 2, 1
  v += ror<0x124>(v);
  v += ror<0x122>(v);
  v += ror<0x121>(v);
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Sums of K values over the W wavefronts of a row.  buf: two halves that calls
// use in turn, so that one barrier per call is enough.
template <int W, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*buf)[W][4], int& turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
  if constexpr (W > 1) {
    const int wv = threadIdx.x / kWave;
    if (threadIdx.x % kWave == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) buf[turn][wv][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) v[k] += buf[turn][w][k];
    }
    turn ^= 1;
  }
}

// A vector of 16 bytes as floats.
template <typename T>
struct Vec {
  static constexpr int N = 16 / static_cast<int>(sizeof(T));
  float f[N];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = 0.0f;
  }
  __device__ __forceinline__ void load(const void* p, int64_t i) { unpack(static_cast<const uint32x4*>(p)[i]); }
  __device__ __forceinline__ void unpack(uint32x4 v) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f[2 * j] = __uint_as_float(v[j] << 16);
        f[2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(v[j]);
    }
  }
  __device__ __forceinline__ void store(void* p, int64_t i) const {
    uint32x4 v;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = pack2(f[2 * j], f[2 * j + 1]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(f[j]);
    }
    static_cast<uint32x4*>(p)[i] = v;
  }
  static __device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, b}, bf16x2));
  }
};

template <typename T>
__device__ __forceinline__ float scalar(const void* p, int64_t i) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
  else return static_cast<const float*>(p)[i];
}

// W wavefronts per row, 4 / W rows (at least one) per workgroup.
template <typename T, int W, int V>
__global__ void __launch_bounds__((W > 4 ? W : 4) * kWave) k_norm(NormArgs a) {
  using X = Vec<T>;
  constexpr int N = X::N;
  constexpr int kRows = W > 4 ? 1 : 4 / W;
  __shared__ float buf[2][W][4];
  int turn = 0;
  const int part = static_cast<int>(threadIdx.x) % (W * kWave);
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / (W * kWave);
  if (t >= a.T) return;   // (whole wavefronts, and no barrier where W < 4)
  const int vecs = a.d / N;
  const int64_t row = t * vecs;
  X r[V];
  bool in[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    in[v] = part + v * W * kWave < vecs;
    r[v].zero();
    if (in[v]) r[v].load(a.x, row + part + v * W * kWave);
  }
  if (a.y != nullptr) {
    X y[V];
    float sum[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      y[v].zero();
      if (in[v]) y[v].load(a.y, row + part + v * W * kWave);
#pragma unroll
      for (int i = 0; i < N; ++i) sum[0] += y[v].f[i] * y[v].f[i];
    }
    float f = a.scale;
    if (a.gate_kind == FM_GATE_TOKEN) f *= scalar<T>(a.gate, t);
    if (a.post != nullptr) {
      row_sums<W, 1>(sum, buf, turn);
      f *= rsqrtf(sum[0] / static_cast<float>(a.d) + a.eps);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!in[v]) continue;
      const int64_t i = part + v * W * kWave;
      X w;
      if (a.post != nullptr) {
        w.load(a.post, i);
#pragma unroll
        for (int j = 0; j < N; ++j) y[v].f[j] *= w.f[j];
      }
      if (a.gate_kind == FM_GATE_CHANNEL || a.gate_kind == FM_GATE_EACH) {
        w.load(a.gate, a.gate_kind == FM_GATE_EACH ? row + i : i);
#pragma unroll
        for (int j = 0; j < N; ++j) y[v].f[j] *= w.f[j];
      }
#pragma unroll
      for (int j = 0; j < N; ++j) r[v].f[j] += f * y[v].f[j];
    }
  }
  if (a.r_out != nullptr) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (in[v]) r[v].store(a.r_out, row + part + v * W * kWave);
  }
  if (a.pre == nullptr) return;
  float sum[1] = {0.0f};
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < N; ++j) sum[0] += r[v].f[j] * r[v].f[j];
  row_sums<W, 1>(sum, buf, turn);
  const float f = rsqrtf(sum[0] / static_cast<float>(a.d) + a.eps);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (!in[v]) continue;
    const int64_t i = part + v * W * kWave;
    X w;
    w.load(a.pre, i);
#pragma unroll
    for (int j = 0; j < N; ++j) w.f[j] *= r[v].f[j] * f;
    w.store(a.h_out, row + i);
  }
}

// The gradient.  A workgroup takes every gridDim.x-th row (of kRows) and keeps its
// share of the sums over rows in registers: dpost, dpre, dgate of a channel.
template <typename T, int W, int V>
__global__ void __launch_bounds__((W > 4 ? W : 4) * kWave) k_norm_grad(NormGradArgs a) {
  using X = Vec<T>;
  constexpr int N = X::N;
  constexpr int kRows = W > 4 ? 1 : 4 / W;
  __shared__ float buf[2][W][4];
  int turn = 0;
  const NormArgs& f = a.f;
  const int part = static_cast<int>(threadIdx.x) % (W * kWave);
  const int vecs = f.d / N;
  const float inv_d = 1.0f / static_cast<float>(f.d);
  bool in[V];
  X post[V], pre[V], sum_post[V], sum_pre[V], sum_gate[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int64_t i = part + v * W * kWave;
    in[v] = i < vecs;
    post[v].zero();
    pre[v].zero();
    sum_post[v].zero();
    sum_pre[v].zero();
    sum_gate[v].zero();
    if (in[v] && f.post != nullptr) post[v].load(f.post, i);
    if (in[v] && f.pre != nullptr) pre[v].load(f.pre, i);
  }
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / (W * kWave); t < f.T;
       t += static_cast<int64_t>(gridDim.x) * kRows) {
    const int64_t row = t * vecs;
    X r[V], y[V], dr[V], dh[V], gate[V];
    float s0[1] = {0.0f};
    const float token = f.gate_kind == FM_GATE_TOKEN ? scalar<T>(f.gate, t) : 1.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int64_t i = part + v * W * kWave;
      r[v].zero();
      y[v].zero();
      dr[v].zero();
      dh[v].zero();
#pragma unroll
      for (int j = 0; j < N; ++j) gate[v].f[j] = token;
      if (!in[v]) continue;
      r[v].load(f.x, row + i);
      if (f.y != nullptr) y[v].load(f.y, row + i);
      if (a.dr != nullptr) dr[v].load(a.dr, row + i);
      if (a.dh != nullptr) dh[v].load(a.dh, row + i);
      if (f.gate_kind == FM_GATE_CHANNEL) gate[v].load(f.gate, i);
      if (f.gate_kind == FM_GATE_EACH) gate[v].load(f.gate, row + i);
#pragma unroll
      for (int j = 0; j < N; ++j) s0[0] += y[v].f[j] * y[v].f[j];
    }
    float inv_y = 1.0f;
    if (f.post != nullptr) {
      row_sums<W, 1>(s0, buf, turn);
      inv_y = rsqrtf(s0[0] * inv_d + f.eps);
    }
    // r = x + scale gate n; sums of r^2 and of dz r
    float s1[2] = {0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        y[v].f[j] *= inv_y;   // normed
        const float n = f.post != nullptr ? y[v].f[j] * post[v].f[j] : y[v].f[j];
        r[v].f[j] += f.scale * gate[v].f[j] * n;
        s1[0] += r[v].f[j] * r[v].f[j];
        s1[1] += dh[v].f[j] * pre[v].f[j] * r[v].f[j];
      }
    if (f.pre != nullptr) {
      row_sums<W, 2>(s1, buf, turn);
      const float inv_r = rsqrtf(s1[0] * inv_d + f.eps);
      const float mean = s1[1] * inv_r * inv_d;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float r_hat = r[v].f[j] * inv_r;
          sum_pre[v].f[j] += dh[v].f[j] * r_hat;
          dr[v].f[j] += inv_r * (dh[v].f[j] * pre[v].f[j] - r_hat * mean);
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (in[v]) dr[v].store(a.dx, row + part + v * W * kWave);
    if (f.y == nullptr) continue;
    // dn into dr, dgate summed or written; sums of dz' y^ and of dgate
    float s2[2] = {0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      X each;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float n = f.post != nullptr ? y[v].f[j] * post[v].f[j] : y[v].f[j];
        const float d = f.scale * dr[v].f[j];
        each.f[j] = d * n;
        sum_gate[v].f[j] += each.f[j];
        s2[1] += each.f[j];
        dr[v].f[j] = d * gate[v].f[j];
        sum_post[v].f[j] += dr[v].f[j] * y[v].f[j];
        s2[0] += dr[v].f[j] * post[v].f[j] * y[v].f[j];
      }
      if (f.gate_kind == FM_GATE_EACH && in[v]) each.store(a.dgate, row + part + v * W * kWave);
    }
    if (f.post != nullptr || f.gate_kind == FM_GATE_TOKEN) row_sums<W, 2>(s2, buf, turn);
    if (f.gate_kind == FM_GATE_TOKEN && part == 0) static_cast<float*>(a.dgate)[t] = s2[1];
    const float mean = s2[0] * inv_d;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (f.post != nullptr) {
#pragma unroll
        for (int j = 0; j < N; ++j) dr[v].f[j] = inv_y * (dr[v].f[j] * post[v].f[j] - y[v].f[j] * mean);
      }
      if (in[v]) dr[v].store(a.dy, row + part + v * W * kWave);
    }
  }
  // this row slot's sums: [gridDim.x * kRows][3][d]
  float* out = a.partial + (static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / (W * kWave)) * 3 * f.d;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (!in[v]) continue;
    const int64_t i = static_cast<int64_t>(part + v * W * kWave) * N;
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      auto put = [&](int which, const X& s) __attribute__((always_inline)) {
        *reinterpret_cast<floatx4*>(out + static_cast<int64_t>(which) * f.d + i + j) =
            floatx4{s.f[j], s.f[j + 1], s.f[j + 2], s.f[j + 3]};
      };
      if (a.dpost != nullptr) put(0, sum_post[v]);
      if (f.gate_kind == FM_GATE_CHANNEL) put(1, sum_gate[v]);
      if (a.dpre != nullptr) put(2, sum_pre[v]);
    }
  }
}

// The sums over the row slots, 64 columns of one gradient per workgroup.
constexpr int kSumWaves = 16;
__global__ void __launch_bounds__(kSumWaves* kWave) k_norm_sum(const float* partial, int32_t lists, int32_t d,
                                                               float* dpost, float* dgate, float* dpre,
                                                               int32_t accumulate) {
  __shared__ float sums[kSumWaves][kWave];
  const int lane = threadIdx.x % kWave;
  const int wv = threadIdx.x / kWave;
  const int which = blockIdx.y;
  float* to = which == 0 ? dpost : (which == 1 ? dgate : dpre);
  if (to == nullptr) return;
  const int col = static_cast<int>(blockIdx.x) * kWave + lane;
  float v = 0.0f;
  if (col < d) {
#pragma unroll 4
    for (int i = wv; i < lists; i += kSumWaves) v += partial[(static_cast<int64_t>(i) * 3 + which) * d + col];
  }
  sums[wv][lane] = v;
  __syncthreads();
  if (wv != 0 || col >= d) return;
  float all = accumulate != 0 ? to[col] : 0.0f;
#pragma unroll
  for (int w = 0; w < kSumWaves; ++w) all += sums[w][lane];
  to[col] = all;
}

// Wavefronts per row and vectors per thread for rows of `vecs` vectors: the fewest
// wavefronts that hold the row with at most VMAX vectors each.
template <typename T>
hipError_t norm(const NormArgs& a, hipStream_t st) {
  const int vecs = a.d / Vec<T>::N;
  auto go = [&](auto w, auto v) {
    constexpr int W = decltype(w)::value, V = decltype(v)::value;
    constexpr int kRows = W > 4 ? 1 : 4 / W;
    const int64_t grid = (static_cast<int64_t>(a.T) + kRows - 1) / kRows;
    k_norm<T, W, V><<<static_cast<unsigned>(grid), (W > 4 ? W : 4) * kWave, 0, st>>>(a);
  };
  using std::integral_constant;
  if (vecs <= kWave) go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
  else if (vecs <= 2 * kWave) go(integral_constant<int, 1>{}, integral_constant<int, 2>{});
  else if (vecs <= 4 * kWave) go(integral_constant<int, 1>{}, integral_constant<int, 4>{});
  else if (vecs <= 8 * kWave) go(integral_constant<int, 4>{}, integral_constant<int, 2>{});
  else if (vecs <= 16 * kWave) go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
  else if (vecs <= 32 * kWave) go(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  else go(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  return hipGetLastError();
}

template <typename T>
hipError_t norm_grad(const NormGradArgs& a, hipStream_t st) {
  const int vecs = a.f.d / Vec<T>::N;
  constexpr int VM = sizeof(T) == 2 ? 2 : 4;   // 16 values of every array per thread
  int lists = 0;
  auto go = [&](auto w, auto v) {
    constexpr int W = decltype(w)::value, V = decltype(v)::value;
    constexpr int kRows = W > 4 ? 1 : 4 / W;
    const int64_t want = (static_cast<int64_t>(a.f.T) + kRows - 1) / kRows;
    const int64_t most = norm_grad_lists(a.f.d) / kRows;
    const unsigned grid = static_cast<unsigned>(want < most ? want : most);
    lists = static_cast<int>(grid) * kRows;
    if (grid > 0) k_norm_grad<T, W, V><<<grid, (W > 4 ? W : 4) * kWave, 0, st>>>(a);
  };
  using std::integral_constant;
  if (vecs <= kWave) go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
  else if (vecs <= VM * kWave) go(integral_constant<int, 1>{}, integral_constant<int, VM>{});
  else if (vecs <= 4 * VM * kWave) go(integral_constant<int, 4>{}, integral_constant<int, VM>{});
  else if (vecs <= 8 * VM * kWave) go(integral_constant<int, 8>{}, integral_constant<int, VM>{});
  else go(integral_constant<int, 16>{}, integral_constant<int, VM>{});
  const bool channel = a.f.gate_kind == FM_GATE_CHANNEL;
  if (a.dpost != nullptr || a.dpre != nullptr || channel)
    k_norm_sum<<<dim3(static_cast<unsigned>((a.f.d + kWave - 1) / kWave), 3), kSumWaves * kWave, 0, st>>>(
        a.partial, lists, a.f.d, a.dpost, channel ? static_cast<float*>(a.dgate) : nullptr, a.dpre, a.accumulate);
  return hipGetLastError();
}

}  // namespace

int norm_grad_lists(int32_t d) { return d <= 1024 ? 2048 : 512; }

size_t norm_scratch_bytes(int32_t T_max, int32_t d) {
  const int64_t most = norm_grad_lists(d);
  const int64_t rows = (static_cast<int64_t>(T_max) + 3) / 4 * 4;
  const int64_t lists = rows < most ? rows : most;
  return align_up(static_cast<size_t>(lists > 0 ? lists : 1) * 3 * static_cast<size_t>(d) * sizeof(float), kAlign);
}

hipError_t launch_norm(const NormArgs& a, fm_dtype dt, hipStream_t st) {
  return dt == FM_BF16 ? norm<uint16_t>(a, st) : norm<float>(a, st);
}

hipError_t launch_norm_grad(const NormGradArgs& a, fm_dtype dt, hipStream_t st) {
  return dt == FM_BF16 ? norm_grad<uint16_t>(a, st) : norm_grad<float>(a, st);
}

}  // namespace fm
