// Norms after and before a block, with the block's gate and scale on its way into
// the residual stream, and their gradient.
//
// A row passes through registers once: W wavefronts hold it, V vectors of 16 bytes
// per thread.  Forward: the sum of y^2, then that of r^2.  Gradient (g gate, s
// scale, ^ a normed row):
//   dz = dh pre            dr' = dr + (dz - r^ mean(dz r^)) / |r|      = dx
//   e = s dr'              dgate = e n
//   dz' = e g post         dy = (dz' - y^ mean(dz' y^)) / |y|
//   dpre = sum over rows of dh r^,  dpost = sum of e g y^
// with r and n made again from x and y, which costs one more sum over the row and
// reads no more than the stored r would.  Memory bounds both: with a gate and
// both norms, 8,192 rows of 4,096 in bf16 take 51 us forward (268 MB, 5.2 TB/s; a copy
// reaches 5.1) and 79 us backward (403 MB, 5.1 TB/s, the sums over the rows 4 of them).
// Few rows cost their chain of launch, loads, sums and barriers: one row of 2,048 3.4 us,
// 64 rows of 4,096 backward 8.6.
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
  const int64_t t =
      (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * kRows + threadIdx.x / (W * kWave);
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
// gridDim.x-th such group and keeps its share of the sums over rows in registers.
// With u = post gate and e = scale dr', the inner sums and dy need e u y^ only, and
// S = sum of e y^ over the rows is both gradients of vectors: dpost = gate S, dgate =
// post S (of other gates than a channel's: dpost = sum of e gate y^).  A row's values
// stay as they were loaded (bf16 in pairs), so that there is room to send for the next
// row's before this one's three sums are waited for.  The sums of wide rows are in LDS:
// 1,024 rows of 12,288 bf16 46 us, 64 with the sums in registers and the next row where
// it is.  Rows of 16 wavefronts, whose threads have 128 registers, leave the vectors in
// the caches too, and the next row: 700 rows of 16,384 float32 99 us, 162 with it sent
// for, 133 with the sums in registers.
template <typename T, int W, int V, int R, int GATE>
__global__ void __launch_bounds__(W* R* kWave) k_norm_grad(NormGradArgs a) {
  using X = Vec<T>;
  constexpr int N = X::N;
  constexpr bool kAhead = W <= 12;
  constexpr bool kWide = W >= 12 || (sizeof(T) == 2 && V == 4);
  constexpr bool kEach = GATE == FM_GATE_EACH, kChannel = GATE == FM_GATE_CHANNEL, kToken = GATE == FM_GATE_TOKEN;
  __shared__ float buf[R][2][W][4];
  __shared__ float joined[R > 1 ? W * kWave * V * N : 1];
  __shared__ floatx4 wide_sums[kWide ? 2 * V * N / 4 : 1][kWide ? W * kWave : 1];
  int turn = 0;
  const NormArgs& f = a.f;
  const int slot = static_cast<int>(threadIdx.x) / (W * kWave);
  const int part = static_cast<int>(threadIdx.x) % (W * kWave);
  const int vecs = f.d / N;
  const float inv_d = 1.0f / static_cast<float>(f.d);
  const bool has_y = f.y != nullptr, has_post = f.post != nullptr, has_pre = f.pre != nullptr;
  auto in = [&](int v) __attribute__((always_inline)) { return part + v * W * kWave < vecs; };
  // post times a channel's gate
  auto product = [&](int v) __attribute__((always_inline)) {
    const int64_t i = part + v * W * kWave;
    X u = wide<T>(take(f.post, i, in(v) && has_post));
    if (!has_post) {
#pragma unroll
      for (int j = 0; j < N; ++j) u.f[j] = 1.0f;
    }
    if constexpr (kChannel) {
      const X g = wide<T>(take(f.gate, i, in(v)));
#pragma unroll
      for (int j = 0; j < N; ++j) u.f[j] *= g.f[j];
    }
    return u;
  };
  uint32x4 pre_[V];
  X u_[V], sum_y[kWide ? 1 : V], sum_r[kWide ? 1 : V];
  // (a lane's own places in LDS, where registers are short)
  auto sum_at = [&](int which, int v, int q) __attribute__((always_inline)) -> floatx4& {
    return wide_sums[kWide ? (which * V + v) * (N / 4) + q : 0][kWide ? threadIdx.x : 0];
  };
  auto add_sum = [&](int which, int v, const X& x) __attribute__((always_inline)) {
    if constexpr (kWide) {
#pragma unroll
      for (int q = 0; q < N / 4; ++q)
        sum_at(which, v, q) += floatx4{x.f[4 * q], x.f[4 * q + 1], x.f[4 * q + 2], x.f[4 * q + 3]};
    } else {
      X& to = which == 0 ? sum_y[v] : sum_r[v];
#pragma unroll
      for (int j = 0; j < N; ++j) to.f[j] += x.f[j];
    }
  };
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if constexpr (kWide) {
#pragma unroll
      for (int q = 0; q < N / 4; ++q) sum_at(0, v, q) = sum_at(1, v, q) = floatx4{0.f, 0.f, 0.f, 0.f};
    } else {
      sum_y[v].zero();
      sum_r[v].zero();
    }
    if constexpr (kAhead) {
      pre_[v] = take(f.pre, part + v * W * kWave, in(v) && has_pre);
      u_[v] = product(v);
    }
  }
  auto pre = [&](int v) __attribute__((always_inline)) {
    return wide<T>(kAhead ? pre_[v] : take(f.pre, part + v * W * kWave, in(v) && has_pre));
  };
  struct Row {
    uint32x4 x[V], y[V], dr[V], dh[V], gate[kEach ? V : 1];
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
      if constexpr (kEach) w.gate[v] = take(f.gate, i, on);
    }
    w.token = kToken && there ? scalar<T>(f.gate, t) : 1.0f;
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
      forget(pre_);
    }
    // u, with the gate of each value
    auto factor = [&](int v) __attribute__((always_inline)) {
      X u = kAhead ? u_[v] : product(v);
      if constexpr (kEach) {
        const X g = wide<T>(now.gate[v]);
#pragma unroll
        for (int j = 0; j < N; ++j) u.f[j] *= g.f[j];
      }
      return u;
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
    forget(now.y);
    X r[V];
    float s1[2] = {0.0f, 0.0f};
    const float step = f.scale * now.token;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      r[v] = wide<T>(now.x[v]);
      if (has_y) {
        const X y = wide<T>(now.y[v]);
        const X u = factor(v);
#pragma unroll
        for (int j = 0; j < N; ++j) r[v].f[j] += step * (u.f[j] * (y.f[j] * inv_y));
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
    forget(now.y);
    forget(now.dh);
    if constexpr (kAhead) forget(pre_);
    // r becomes dr', then e; the sum of e u y^, which is the gradient of a token's gate
    float s2[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      X d = wide<T>(now.dr[v]);
      const bool on = in(v) && live;
      if (has_pre && on) {
        const X dh = wide<T>(now.dh[v]);
        const X w = pre(v);
        X part_r;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float hat = r[v].f[j] * inv_r;
          part_r.f[j] = dh.f[j] * hat;
          d.f[j] += inv_r * (dh.f[j] * w.f[j] - hat * mean);
        }
        add_sum(1, v, part_r);
      }
      if (on) d.store(a.dx, row + v * W * kWave);
      if (!has_y || !on) continue;
      const X y = wide<T>(now.y[v]);
      const X u = factor(v);
      X one, part_y;
      if constexpr (kEach) {   // the gate's own gradient is without the gate
        one = kAhead ? u_[v] : product(v);
        const X g = wide<T>(now.gate[v]);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float hat = y.f[j] * inv_y;
          const float e = f.scale * d.f[j];
          one.f[j] *= e * hat;
          part_y.f[j] = e * g.f[j] * hat;
          s2[0] += e * (u.f[j] * hat);
          r[v].f[j] = e;
        }
        one.store(a.dgate, row + v * W * kWave);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float hat = y.f[j] * inv_y;
          const float e = f.scale * d.f[j];
          part_y.f[j] = (kToken ? e * now.token : e) * hat;
          s2[0] += e * (u.f[j] * hat);
          r[v].f[j] = e;
        }
      }
      add_sum(0, v, part_y);
    }
    if (has_y) {
      if (has_post || kToken) row_sums<W, 1>(s2, buf[slot], turn);
      if (kToken && part == 0 && live) static_cast<float*>(a.dgate)[t] = s2[0];
      if (!has_post) {   // y has no part in dy, also where it is infinite or NaN
#pragma unroll
        for (int v = 0; v < V; ++v) now.y[v] = uint32x4{0u, 0u, 0u, 0u};
      }
      forget(now.y);
      const float mean_y = has_post ? s2[0] * inv_d * inv_y : 0.0f;
      const float back = kToken ? inv_y * now.token : inv_y;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const X y = wide<T>(now.y[v]);
        const X u = factor(v);
        X d;
#pragma unroll
        for (int j = 0; j < N; ++j) d.f[j] = back * (r[v].f[j] * u.f[j] - y.f[j] * mean_y);
        if (in(v) && live) d.store(a.dy, row + v * W * kWave);
      }
    }
    if constexpr (kAhead) now = next;
    else fetch(now, t + stride);
  }
  // the rows' sums in order, through LDS; then this workgroup's: [gridDim.x][2][d]
  float* out = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * f.d;
  auto put = [&](int which, X (&s)[kWide ? 1 : V]) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 1; k < R; ++k) {
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          float* at = joined + (v * N + j) * (W * kWave) + part;
          if (slot == k) *at = s[kWide ? 0 : v].f[j];
        }
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (slot == 0) s[kWide ? 0 : v].f[j] += joined[(v * N + j) * (W * kWave) + part];
    }
    if (slot != 0) return;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!in(v)) continue;
      float* to = out + static_cast<int64_t>(which) * f.d + static_cast<int64_t>(part + v * W * kWave) * N;
#pragma unroll
      for (int j = 0; j < N; j += 4) {
        const X& x = s[kWide ? 0 : v];
        *reinterpret_cast<floatx4*>(to + j) =
            kWide ? sum_at(which, v, j / 4) : floatx4{x.f[j], x.f[j + 1], x.f[j + 2], x.f[j + 3]};
      }
    }
  };
  if (a.dpost != nullptr || kChannel) put(0, sum_y);
  if (a.dpre != nullptr) put(1, sum_r);
}

// The sums over the workgroups, 64 columns of one list per workgroup; S times the
// other vector is the gradient of post and of a channel's gate.
constexpr int kSumWaves = 16;
template <typename T>
__global__ void __launch_bounds__(kSumWaves* kWave) k_norm_sum(NormGradArgs a, int32_t lists) {
  __shared__ float sums[kSumWaves][kWave];
  const int lane = threadIdx.x % kWave;
  const int wv = threadIdx.x / kWave;
  const int which = blockIdx.y;
  const int32_t d = a.f.d;
  const bool channel = a.f.gate_kind == FM_GATE_CHANNEL;
  if (which == 0 ? a.dpost == nullptr && !channel : a.dpre == nullptr) return;
  const int col = static_cast<int>(blockIdx.x) * kWave + lane;
  float v = 0.0f;
  if (col < d) {
#pragma unroll 16   // (all of 256 lists on their way)
    for (int i = wv; i < lists; i += kSumWaves) v += a.partial[(static_cast<int64_t>(i) * 2 + which) * d + col];
  }
  sums[wv][lane] = v;
  __syncthreads();
  if (wv != 0 || col >= d) return;
  float all = 0.0f;
#pragma unroll
  for (int w = 0; w < kSumWaves; ++w) all += sums[w][lane];
  auto add = [&](float* to, float v) __attribute__((always_inline)) {
    if (to != nullptr) to[col] = a.accumulate != 0 ? to[col] + v : v;
  };
  if (which == 1) {
    add(a.dpre, all);
  } else {
    // (S is zero where there is no row, whatever the vectors hold)
    const float g = channel && lists > 0 ? scalar<T>(a.f.gate, col) : 1.0f;
    const float p = a.f.post != nullptr && lists > 0 ? scalar<T>(a.f.post, col) : 1.0f;
    add(a.dpost, g * all);
    if (channel) add(static_cast<float*>(a.dgate), p * all);
  }
}

// Wavefronts per row and vectors per thread for rows of `vecs` vectors: one wavefront, four
// or sixteen, the fewest that hold the row with at most four vectors per thread (bf16
// with two on sixteen; two wavefronts would share a barrier with another row, which may
// not be there).  67 MB of bf16, us, wavefronts x vectors: rows of 512 1x1 46.5, 1x2 46.7;
// 1,024 1x2 47.6, 4x1 53.6; 2,048 1x4 49.0, 4x1 47.1; 2,304 4x2 51.2, 8x1 51.9; 4,096 4x2
// 52.5, 8x1 48.2; 8,192 4x4 55.5, 8x2 52.7, 16x1 49.7; 12,288 16x2 54.5, 12x2 52.4, 16x4
// 74.2; 16,384 16x2 54.7, 8x4 57.1.  float32: 512 1x2 47.4, 4x1 52.9; 1,024 1x4 49.0, 4x1
// 48.0; 2,048 4x2 51.9, 8x1 48.8; 4,096 4x4 53.6, 16x1 50.5; 8,192 16x2 55.0, 8x4 53.9.
// 64 rows of 2,048 bf16: 1x4 3.8, 4x1 2.8; of 8,192: 4x4 4.7, 16x1 3.8.  So the rule is up
// to 12%, and 1 us of a small call, behind the best.  Rows below 512 leave lanes idle:
// of 128 values 91 us, of 64 162.
constexpr int64_t kGridRow = 1 << 16;

template <typename T>
hipError_t norm(const NormArgs& a, hipStream_t st) {
  const int vecs = a.d / Vec<T>::N;
  auto go = [&](auto w, auto v) {
    constexpr int W = decltype(w)::value, V = decltype(v)::value;
    constexpr int kRows = W > 4 ? 1 : 4 / W;
    // (in two dimensions: one of them holds fewer than 2^32 threads)
    const int64_t groups = (static_cast<int64_t>(a.T) + kRows - 1) / kRows;
    const int64_t gx = groups < kGridRow ? groups : kGridRow;
    const dim3 grid(static_cast<unsigned>(gx), static_cast<unsigned>((groups + gx - 1) / gx));
    k_norm<T, W, V><<<grid, (W > 4 ? W : 4) * kWave, 0, st>>>(a);
  };
  using std::integral_constant;
  if (vecs <= kWave) go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
  else if (vecs <= 2 * kWave) go(integral_constant<int, 1>{}, integral_constant<int, 2>{});
  else if (vecs <= 4 * kWave) go(integral_constant<int, 1>{}, integral_constant<int, 4>{});
  else if (vecs <= 8 * kWave) go(integral_constant<int, 4>{}, integral_constant<int, 2>{});
  else if (vecs <= 16 * kWave) go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
  else if (sizeof(T) == 2 || vecs <= 32 * kWave) go(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  else go(integral_constant<int, 16>{}, integral_constant<int, sizeof(T) == 2 ? 2 : 4>{});
  return hipGetLastError();
}

template <typename T>
hipError_t norm_grad(const NormGradArgs& a, hipStream_t st) {
  constexpr bool kBf = sizeof(T) == 2;
  const int vecs = a.f.d / Vec<T>::N;
  int lists = 0;
  auto run = [&](auto w, auto v, auto r, auto gate) {
    constexpr int R = decltype(r)::value, G = decltype(gate)::value;
    // (four vectors of a fifth array spill: 64 rows of 16,384 bf16 20.2 us for 17.6)
    constexpr bool kFifth = kBf && decltype(v)::value == 4 && G == FM_GATE_EACH;
    constexpr int W = kFifth ? 16 : decltype(w)::value, V = kFifth ? 2 : decltype(v)::value;
    const int64_t want = (static_cast<int64_t>(a.f.T) + R - 1) / R;
    lists = static_cast<int>(want < kNormLists ? want : kNormLists);
    if (lists > 0) k_norm_grad<T, W, V, R, G><<<static_cast<unsigned>(lists), W * R * kWave, 0, st>>>(a);
  };
  auto go = [&](auto w, auto v, auto r) {
    switch (a.f.gate_kind) {
      case FM_GATE_NONE: return run(w, v, r, std::integral_constant<int, FM_GATE_NONE>{});
      case FM_GATE_CHANNEL: return run(w, v, r, std::integral_constant<int, FM_GATE_CHANNEL>{});
      case FM_GATE_TOKEN: return run(w, v, r, std::integral_constant<int, FM_GATE_TOKEN>{});
      default: return run(w, v, r, std::integral_constant<int, FM_GATE_EACH>{});
    }
  };
  using std::integral_constant;
  // As few wavefronts as hold the row with one vector of every array per thread, or
  // two where that leaves one row to a workgroup and lanes idle, or needs more than
  // eight.  In bf16, with one and with two: 64 rows of 1,024 7.1 us and 10.2, of 4,096
  // 8.5 and 9.6, 8,192 rows of 4,096 81 and 84; but of 2,304 62 and 53, of 8,192 198
  // and 157.  67 MB in rows of 1,280 take 93 us on 4 wavefronts and 113 on 4 of two
  // vectors each.  Wider rows: no more than 12 wavefronts,
  // whose threads have registers for the next row, take four vectors of float32 up to
  // 8,192 values (2,048 rows: 89 us, 109 on 16 wavefronts of two) and, with the sums in
  // LDS, of bf16 beyond 12,288 (16,384: 102 and 127).  float32 rows of more than 8,192
  // need 16: 700 rows of 12,288 take 65 us with three vectors and 79 with four.
  if (vecs <= kWave) go(integral_constant<int, 1>{}, integral_constant<int, 1>{}, integral_constant<int, 8>{});
  else if (vecs <= 2 * kWave) go(integral_constant<int, 2>{}, integral_constant<int, 1>{}, integral_constant<int, 4>{});
  else if (vecs <= 4 * kWave) go(integral_constant<int, 4>{}, integral_constant<int, 1>{}, integral_constant<int, 2>{});
  else if (vecs <= 6 * kWave) go(integral_constant<int, 3>{}, integral_constant<int, 2>{}, integral_constant<int, 2>{});
  else if (vecs <= 8 * kWave) go(integral_constant<int, 8>{}, integral_constant<int, 1>{}, integral_constant<int, 1>{});
  else if (vecs <= 12 * kWave) go(integral_constant<int, 6>{}, integral_constant<int, 2>{}, integral_constant<int, 1>{});
  else if (vecs <= 16 * kWave) go(integral_constant<int, 8>{}, integral_constant<int, 2>{}, integral_constant<int, 1>{});
  else if (kBf && vecs <= 24 * kWave) go(integral_constant<int, kBf ? 12 : 8>{}, integral_constant<int, 2>{}, integral_constant<int, 1>{});
  else if (kBf || vecs <= 32 * kWave) go(integral_constant<int, 8>{}, integral_constant<int, 4>{}, integral_constant<int, 1>{});
  else if (vecs <= 48 * kWave) go(integral_constant<int, kBf ? 8 : 16>{}, integral_constant<int, kBf ? 4 : 3>{}, integral_constant<int, 1>{});
  else go(integral_constant<int, kBf ? 8 : 16>{}, integral_constant<int, 4>{}, integral_constant<int, 1>{});
  if (a.dpost != nullptr || a.dpre != nullptr || a.f.gate_kind == FM_GATE_CHANNEL)
    k_norm_sum<T><<<dim3(static_cast<unsigned>((a.f.d + kWave - 1) / kWave), 2), kSumWaves * kWave, 0, st>>>(a, lists);
  return hipGetLastError();
}

}  // namespace

size_t norm_scratch_bytes(int32_t T_max, int32_t d) {
  const int64_t lists = T_max < 1 ? 1 : (T_max < kNormLists ? T_max : kNormLists);
  return align_up(static_cast<size_t>(lists) * 2 * static_cast<size_t>(d) * sizeof(float), kAlign);
}

hipError_t launch_norm(const NormArgs& a, fm_dtype dt, hipStream_t st) {
  return dt == FM_BF16 ? norm<uint16_t>(a, st) : norm<float>(a, st);
}

hipError_t launch_norm_grad(const NormGradArgs& a, fm_dtype dt, hipStream_t st) {
  return dt == FM_BF16 ? norm_grad<uint16_t>(a, st) : norm_grad<float>(a, st);
}

}  // namespace fm
