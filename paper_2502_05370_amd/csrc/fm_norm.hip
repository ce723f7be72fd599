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
    const int wv = threadIdx.x / kWave % W;
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

// Sixteen bytes of a row or a vector, zeros where there are none.
__device__ __forceinline__ uint32x4 take(const void* p, int64_t i, bool there) {
  return there ? static_cast<const uint32x4*>(p)[i] : uint32x4{0u, 0u, 0u, 0u};
}
template <typename T>
__device__ __forceinline__ Vec<T> wide(uint32x4 v) {
  Vec<T> w;
  w.unpack(v);
  return w;
}

// The compiler keeps what it unpacked from v before, or outside a loop, no longer:
// registers for floats beside the bf16 pairs that they come from.
template <int V>
__device__ __forceinline__ void forget(uint32x4 (&v)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) asm volatile("" : "+v"(v[i]));
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
  const bool each = a.gate_kind == FM_GATE_EACH;
  // all that the row needs is sent for before anything waits
  uint32x4 xp[V], yp[V], gp[V], post[V], pre[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int64_t i = part + v * W * kWave;
    const bool in = i < vecs;
    yp[v] = take(a.y, row + i, in && a.y != nullptr);
    xp[v] = take(a.x, row + i, in);
    gp[v] = take(a.gate, each ? row + i : i, in && (each || a.gate_kind == FM_GATE_CHANNEL));
    post[v] = take(a.post, i, in && a.post != nullptr);
    pre[v] = take(a.pre, i, in && a.pre != nullptr);
  }
  const float token = a.gate_kind == FM_GATE_TOKEN ? scalar<T>(a.gate, t) : 1.0f;
  float f = 1.0f;
  if (a.post != nullptr) {
    float sum[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const X y = wide<T>(yp[v]);
#pragma unroll
      for (int j = 0; j < N; ++j) sum[0] += y.f[j] * y.f[j];
    }
    row_sums<W, 1>(sum, buf, turn);
    f = rsqrtf(sum[0] / static_cast<float>(a.d) + a.eps);
  }
  f *= a.scale * token;
  X r[V];
  float sum[1] = {0.0f};
#pragma unroll
  for (int v = 0; v < V; ++v) {
    r[v] = wide<T>(xp[v]);
    if (a.y != nullptr) {
      X n = wide<T>(yp[v]);
      if (a.post != nullptr) {
        const X w = wide<T>(post[v]);
#pragma unroll
        for (int j = 0; j < N; ++j) n.f[j] *= w.f[j];
      }
      if (each || a.gate_kind == FM_GATE_CHANNEL) {
        const X w = wide<T>(gp[v]);
#pragma unroll
        for (int j = 0; j < N; ++j) n.f[j] *= w.f[j];
      }
#pragma unroll
      for (int j = 0; j < N; ++j) r[v].f[j] += f * n.f[j];
    }
    const int64_t i = part + v * W * kWave;
    if (a.r_out != nullptr && i < vecs) r[v].store(a.r_out, row + i);
    // (past the row f n is zero times zero, or NaN where f is infinite)
#pragma unroll
    for (int j = 0; j < N; ++j) sum[0] += i < vecs ? r[v].f[j] * r[v].f[j] : 0.0f;
  }
  if (a.pre == nullptr) return;
  row_sums<W, 1>(sum, buf, turn);
  f = rsqrtf(sum[0] / static_cast<float>(a.d) + a.eps);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int64_t i = part + v * W * kWave;
    if (i >= vecs) continue;
    X w = wide<T>(pre[v]);
#pragma unroll
    for (int j = 0; j < N; ++j) w.f[j] *= r[v].f[j] * f;
    w.store(a.h_out, row + i);
  }
}

// The gradient.  R rows of W wavefronts per workgroup, which takes every
// gridDim.x-th such group and keeps its share of the sums over rows in registers:
// dpost, dpre, dgate of a channel.  A row's values stay as they were loaded (bf16 in
// pairs), so that there is room to send for the next row's before this one's three
// sums are waited for.  Rows of 16 wavefronts leave the vectors in the caches and the
// next row where it is.
template <typename T, int W, int V, int R>
__global__ void __launch_bounds__(W* R* kWave) k_norm_grad(NormGradArgs a) {
  using X = Vec<T>;
  constexpr int N = X::N;
  constexpr bool kAhead = W <= 8;
  __shared__ float buf[R][2][W][4];
  __shared__ float joined[R > 1 ? W * kWave * V * N : 1];
  int turn = 0;
  const NormArgs& f = a.f;
  const int slot = static_cast<int>(threadIdx.x) / (W * kWave);
  const int part = static_cast<int>(threadIdx.x) % (W * kWave);
  const int vecs = f.d / N;
  const float inv_d = 1.0f / static_cast<float>(f.d);
  const bool each = f.gate_kind == FM_GATE_EACH, channel = f.gate_kind == FM_GATE_CHANNEL;
  const bool has_y = f.y != nullptr, has_post = f.post != nullptr, has_pre = f.pre != nullptr;
  uint32x4 post_[V], pre_[V], gate_[V];
  X sum_post[V], sum_pre[V], sum_gate[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int64_t i = part + v * W * kWave;
    sum_post[v].zero();
    sum_pre[v].zero();
    sum_gate[v].zero();
    if constexpr (kAhead) {
      post_[v] = take(f.post, i, i < vecs && has_post);
      pre_[v] = take(f.pre, i, i < vecs && has_pre);
      gate_[v] = take(f.gate, i, i < vecs && channel);
    }
  }
  auto in = [&](int v) __attribute__((always_inline)) { return part + v * W * kWave < vecs; };
  auto post = [&](int v) __attribute__((always_inline)) {
    return wide<T>(kAhead ? post_[v] : take(f.post, part + v * W * kWave, in(v) && has_post));
  };
  auto pre = [&](int v) __attribute__((always_inline)) {
    return wide<T>(kAhead ? pre_[v] : take(f.pre, part + v * W * kWave, in(v) && has_pre));
  };
  struct Row {
    uint32x4 x[V], y[V], dr[V], dh[V], gate[V];
    float token;
  };
  auto fetch = [&](Row& w, int64_t t) __attribute__((always_inline)) {
    const bool there = t < f.T;
    const int64_t row = t * vecs + part;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int64_t i = row + v * W * kWave;
      const bool on = there && in(v);
      w.y[v] = take(f.y, i, on && has_y);
      w.x[v] = take(f.x, i, on);
      w.dh[v] = take(a.dh, i, on && a.dh != nullptr);
      w.dr[v] = take(a.dr, i, on && a.dr != nullptr);
      if (each) w.gate[v] = take(f.gate, i, on);
    }
    w.token = f.gate_kind == FM_GATE_TOKEN && there ? scalar<T>(f.gate, t) : 1.0f;
  };
  const int64_t stride = static_cast<int64_t>(gridDim.x) * R;
  int64_t t = static_cast<int64_t>(blockIdx.x) * R + slot;
  Row now, next;
  fetch(now, t);
  // (the rows of a workgroup meet in barriers: all of it stays until its first row
  // has passed the end)
  for (; t - slot < f.T; t += stride) {
    const bool live = t < f.T;
    const int64_t row = t * vecs + part;
    if constexpr (kAhead) {
      fetch(next, t + stride);
      forget(post_);
      forget(pre_);
      forget(gate_);
    }
    auto gate = [&](int v) __attribute__((always_inline)) {
      X g;
      if (each || channel) {
        if constexpr (kAhead) g = wide<T>(each ? now.gate[v] : gate_[v]);
        else g = wide<T>(each ? now.gate[v] : take(f.gate, part + v * W * kWave, in(v)));
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) g.f[j] = now.token;
      }
      return g;
    };
    float inv_y = 1.0f;
    if (has_post) {
      float s[1] = {0.0f};
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const X y = wide<T>(now.y[v]);
#pragma unroll
        for (int j = 0; j < N; ++j) s[0] += y.f[j] * y.f[j];
      }
      row_sums<W, 1>(s, buf[slot], turn);
      inv_y = rsqrtf(s[0] * inv_d + f.eps);
    }
    auto again = [&]() __attribute__((always_inline)) {   // between the sums
      forget(now.y);
      forget(now.dh);
      if constexpr (kAhead) {
        forget(post_);
        forget(pre_);
        forget(gate_);
      }
    };
    again();
    // n: y^ post, or y^ where there is no post
    auto normed = [&](int v, X& hat, X& n) __attribute__((always_inline)) {
      hat = wide<T>(now.y[v]);
      const X w = post(v);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        hat.f[j] *= inv_y;
        n.f[j] = has_post ? hat.f[j] * w.f[j] : hat.f[j];
      }
    };
    X r[V];
    float s1[2] = {0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      r[v] = wide<T>(now.x[v]);
      if (has_y) {
        X hat, n;
        normed(v, hat, n);
        const X g = gate(v);
#pragma unroll
        for (int j = 0; j < N; ++j) r[v].f[j] += f.scale * g.f[j] * n.f[j];
      }
      if (!in(v)) r[v].zero();
      const X dh = wide<T>(now.dh[v]);
      const X w = pre(v);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        s1[0] += r[v].f[j] * r[v].f[j];
        s1[1] += dh.f[j] * w.f[j] * r[v].f[j];
      }
    }
    float inv_r = 0.0f, mean = 0.0f;
    if (has_pre) {
      row_sums<W, 2>(s1, buf[slot], turn);
      inv_r = rsqrtf(s1[0] * inv_d + f.eps);
      mean = s1[1] * inv_r * inv_d;
    }
    again();
    // r becomes dr'; then dn, and sums of dz' y^ and of dgate
    float s2[2] = {0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      X d = wide<T>(now.dr[v]);
      if (has_pre && in(v) && live) {
        const X dh = wide<T>(now.dh[v]);
        const X w = pre(v);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float hat = r[v].f[j] * inv_r;
          sum_pre[v].f[j] += dh.f[j] * hat;
          d.f[j] += inv_r * (dh.f[j] * w.f[j] - hat * mean);
        }
      }
      r[v] = d;
      if (in(v) && live) d.store(a.dx, row + v * W * kWave);
      if (!has_y || !in(v) || !live) continue;
      X hat, n;
      normed(v, hat, n);
      const X g = gate(v);
      const X w = post(v);
      X one;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float e = f.scale * d.f[j];
        one.f[j] = e * n.f[j];
        sum_gate[v].f[j] += one.f[j];
        s2[1] += one.f[j];
        const float dn = e * g.f[j];
        sum_post[v].f[j] += dn * hat.f[j];
        s2[0] += dn * w.f[j] * hat.f[j];
        r[v].f[j] = dn;
      }
      if (each) one.store(a.dgate, row + v * W * kWave);
    }
    if (has_y) {
      if (has_post || f.gate_kind == FM_GATE_TOKEN) row_sums<W, 2>(s2, buf[slot], turn);
      if (f.gate_kind == FM_GATE_TOKEN && part == 0 && live) static_cast<float*>(a.dgate)[t] = s2[1];
      again();
      const float mean_y = s2[0] * inv_d;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (has_post) {
          const X y = wide<T>(now.y[v]);
          const X w = post(v);
#pragma unroll
          for (int j = 0; j < N; ++j) r[v].f[j] = inv_y * (r[v].f[j] * w.f[j] - y.f[j] * inv_y * mean_y);
        }
        if (in(v) && live) r[v].store(a.dy, row + v * W * kWave);
      }
    }
    if constexpr (kAhead) now = next;
    else fetch(now, t + stride);
  }
  // the rows' sums in order, through LDS; then this workgroup's: [gridDim.x][3][d]
  float* out = a.partial + static_cast<int64_t>(blockIdx.x) * 3 * f.d;
  auto put = [&](int which, X (&s)[V]) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 1; k < R; ++k) {
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          float* at = joined + (v * N + j) * (W * kWave) + part;
          if (slot == k) *at = s[v].f[j];
        }
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (slot == 0) s[v].f[j] += joined[(v * N + j) * (W * kWave) + part];
    }
    if (slot != 0) return;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!in(v)) continue;
      float* to = out + static_cast<int64_t>(which) * f.d + static_cast<int64_t>(part + v * W * kWave) * N;
#pragma unroll
      for (int j = 0; j < N; j += 4)
        *reinterpret_cast<floatx4*>(to + j) = floatx4{s[v].f[j], s[v].f[j + 1], s[v].f[j + 2], s[v].f[j + 3]};
    }
  };
  if (a.dpost != nullptr) put(0, sum_post);
  if (channel) put(1, sum_gate);
  if (a.dpre != nullptr) put(2, sum_pre);
}

// The sums over the workgroups, 64 columns of one gradient per workgroup.
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
  int lists = 0;
  auto go = [&](auto w, auto v, auto r) {
    constexpr int W = decltype(w)::value, V = decltype(v)::value, R = decltype(r)::value;
    const int64_t want = (static_cast<int64_t>(a.f.T) + R - 1) / R;
    lists = static_cast<int>(want < kNormLists ? want : kNormLists);
    if (lists > 0) k_norm_grad<T, W, V, R><<<static_cast<unsigned>(lists), W * R * kWave, 0, st>>>(a);
  };
  using std::integral_constant;
  // two vectors of every array per thread; four where no more wavefronts can be had
  if (vecs <= kWave) go(integral_constant<int, 1>{}, integral_constant<int, 1>{}, integral_constant<int, 8>{});
  else if (vecs <= 2 * kWave) go(integral_constant<int, 1>{}, integral_constant<int, 2>{}, integral_constant<int, 8>{});
  else if (vecs <= 8 * kWave) go(integral_constant<int, 4>{}, integral_constant<int, 2>{}, integral_constant<int, 2>{});
  else if (vecs <= 16 * kWave) go(integral_constant<int, 8>{}, integral_constant<int, 2>{}, integral_constant<int, 1>{});
  else if (vecs <= 32 * kWave) go(integral_constant<int, 16>{}, integral_constant<int, 2>{}, integral_constant<int, 1>{});
  else go(integral_constant<int, 16>{}, integral_constant<int, 4>{}, integral_constant<int, 1>{});
  const bool channel = a.f.gate_kind == FM_GATE_CHANNEL;
  if (a.dpost != nullptr || a.dpre != nullptr || channel)
    k_norm_sum<<<dim3(static_cast<unsigned>((a.f.d + kWave - 1) / kWave), 3), kSumWaves * kWave, 0, st>>>(
        a.partial, lists, a.f.d, a.dpost, channel ? static_cast<float*>(a.dgate) : nullptr, a.dpre, a.accumulate);
  return hipGetLastError();
}

}  // namespace

size_t norm_scratch_bytes(int32_t T_max, int32_t d) {
  const int64_t lists = T_max < 1 ? 1 : (T_max < kNormLists ? T_max : kNormLists);
  return align_up(static_cast<size_t>(lists) * 3 * static_cast<size_t>(d) * sizeof(float), kAlign);
}

hipError_t launch_norm(const NormArgs& a, fm_dtype dt, hipStream_t st) {
  return dt == FM_BF16 ? norm<uint16_t>(a, st) : norm<float>(a, st);
}

hipError_t launch_norm_grad(const NormGradArgs& a, fm_dtype dt, hipStream_t st) {
  return dt == FM_BF16 ? norm_grad<uint16_t>(a, st) : norm_grad<float>(a, st);
}

}  // namespace fm
