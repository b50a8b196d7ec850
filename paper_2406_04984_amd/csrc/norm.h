// Layer norm and root-mean-square norm of rows, forward and backward, alone or behind dropout and a residual add:
//
//   y = res + drop(out)  (or y = x)       mu = mean y (0 for the rms kind)   r = 1 / sqrt(mean (y - mu)^2 + eps)
//   h = (y - mu) r gamma + beta
//   g = dh gamma,  xh = (y - mu) r:       dy' = r (g - mean g [layer kind] - xh mean(g xh)) + dy
//   dgamma = sum_t dh xh,  dbeta = sum_t dh,  dout = drop(dy')
//
// W waves share a row and hold it in registers, V groups of eight columns per lane: the row is read once, its mean is
// subtracted before the squares are summed, and all sums are fp32.
#pragma once
#include "common.h"
#include "dropout.h"

namespace meft {

// v as it is stored in T
template <typename T>
__device__ __forceinline__ void round8(float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = pack_bf16x2(v[2 * i], v[2 * i + 1]);
      v[2 * i] = __uint_as_float(w << 16);
      v[2 * i + 1] = __uint_as_float(w & 0xFFFF0000u);
    }
  }
}

// Sums over the W waves of a row.  Calls alternate between two buffers, so one barrier each is enough: a wave writes a buffer
// again only behind the barrier of the call in between, which the last reader of the former contents has passed.
template <int W, int kMaxSlots, int kValues>
struct RowSum {
  float* lds;   // [2][kMaxSlots][W][kValues]
  int turn = 0;
  __device__ __forceinline__ void operator()(float (&v)[kValues], int slot, int wave) {
#pragma unroll
    for (int i = 0; i < kValues; ++i) v[i] = wave_sum(v[i]);
    if constexpr (W > 1) {
      float* p = lds + (size_t)((turn * kMaxSlots + slot) * W) * kValues;
      turn ^= 1;
      if ((threadIdx.x & 63) < kValues) {
        float mine = v[0];
#pragma unroll
        for (int i = 1; i < kValues; ++i) mine = (threadIdx.x & 63) == i ? v[i] : mine;
        p[wave * kValues + (threadIdx.x & 63)] = mine;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kValues; ++i) {
        float s = p[i];
#pragma unroll
        for (int w = 1; w < W; ++w) s += p[w * kValues + i];
        v[i] = s;
      }
    }
  }
};

enum { kNormPlain = 0, kNormAdd = 1, kNormDrop = 2 };   // y = x, y = res + out, y = res + drop(out)

template <typename T>
struct NormFwdArgs {
  const T *x, *out, *gamma, *beta;   // x: res where there is an add
  T *y, *h;
  float *mean, *rstd;
  int n_tok, d, layer;
  float inv_d, eps;
  bool past;   // h past L2 (kNormPlain)
  DropArgs drop;
};

// Rows (slots of W waves) of a workgroup of norm_fwd_kernel and norm_bwd_kernel at most; the launch says how many there are.
constexpr int norm_max_slots(int w) { return w >= 4 ? 1 : 4 / w; }

// Memory bounds it.  A row's words are asked for while the row before is computed: they are widened at the top of a round, and
// their registers then take the next row's.  8192 x 4096 bf16, rms: 25 us on average (5.3 TB/s); before
// results went past L2, 24 and 28 with each row asked for when its turn comes.  With dropout and the residual add 53 us for twice
// the bytes.
template <typename T, int V, int W, int kMode>
__global__ __launch_bounds__(64 * W * norm_max_slots(W)) void norm_fwd_kernel(NormFwdArgs<T> a) {
  constexpr int kMaxSlots = norm_max_slots(W);
  __shared__ float s_sum[2 * kMaxSlots * W];
  const int slots = blockDim.x / (64 * W), slot = threadIdx.x / (64 * W), q = threadIdx.x % (64 * W), wave = q / 64;
  RowSum<W, kMaxSlots, 1> row_sum{s_sum};
  const uint64_t offset = kMode == kNormDrop ? drop_offset(a.drop) : 0;
  Raw8<T> gamma[V], beta[V], raw_x[V], raw_out[V];
  bool in[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (i * 64 * W + q) * 8;
    in[i] = c < a.d;
    gamma[i].clear();
    beta[i].clear();
    raw_x[i].clear();
    raw_out[i].clear();
    if (in[i]) gamma[i].load(a.gamma + c);
    if (in[i] && a.beta) beta[i].load(a.beta + c);
  }
  auto load = [&](int64_t t) {
    if (t >= a.n_tok) return;
    const size_t row = (size_t)t * a.d;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * 64 * W + q) * 8;
      if (!in[i]) continue;
      raw_x[i].load(a.x + row + c);
      if (kMode != kNormPlain) raw_out[i].load(a.out + row + c);
    }
  };
  const int64_t stride = (int64_t)gridDim.x * slots;
  load((int64_t)blockIdx.x * slots + slot);
  for (int64_t first = (int64_t)blockIdx.x * slots; first < a.n_tok; first += stride) {
    const int64_t t = first + slot;
    const bool live = t < a.n_tok;
    const size_t row = (size_t)t * a.d;
    float v[V][8], o[V][8];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      raw_x[i].widen(v[i]);
      if (kMode != kNormPlain) raw_out[i].widen(o[i]);
    }
    load(t + stride);
    if (kMode != kNormPlain) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = (i * 64 * W + q) * 8;
        if (kMode == kNormDrop) drop8(a.drop, offset, (uint32_t)t, c / 8, o[i]);
#pragma unroll
        for (int z = 0; z < 8; ++z) v[i][z] += o[i][z];
        round8<T>(v[i]);   // the norm is of the stream as it is stored, which is what the backward reads
        if (live && in[i]) Vec8<T>::store(a.y + row + c, v[i]);
      }
    }
    float mean[1] = {0.f}, sq[1] = {0.f};
    if (a.layer) {
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int z = 0; z < 8; ++z) mean[0] += v[i][z];
      row_sum(mean, slot, wave);
      mean[0] *= a.inv_d;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        const float c = in[i] ? v[i][z] - mean[0] : 0.f;
        sq[0] += c * c;
      }
    row_sum(sq, slot, wave);
    const float rstd = 1.f / sqrtf(sq[0] * a.inv_d + a.eps);
    if (!live) continue;
    if (q == 0) {
      if (a.mean) a.mean[t] = mean[0];
      if (a.rstd) a.rstd[t] = rstd;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (!in[i]) continue;
      float gm[8], bt[8];
      gamma[i].widen(gm);
      beta[i].widen(bt);
#pragma unroll
      for (int z = 0; z < 8; ++z) v[i][z] = (v[i][z] - mean[0]) * rstd * gm[z] + bt[z];
      store8(a.h + row + (i * 64 * W + q) * 8, v[i], kMode == kNormPlain && a.past);
    }
  }
}

template <typename T>
struct NormBwdArgs {
  const T *y, *gamma, *dh, *dy;
  const float *mean, *rstd;
  T *dx, *dout;
  float* part;   // [workgroup][dgamma, dbeta][d]
  T *dgamma, *dbeta;
  int row_wgs;
  int n_tok, d, layer;
  float inv_d;
  bool past;   // dx past L2 (kNormPlain)
  DropArgs drop;
};

// dgamma and dbeta (may be null) of kApartCols columns by one workgroup, over all rows: they need no sums over a
// row.  What bounds it is the 100 or so lines that a compute unit has on their way, so a line holds as many of its columns as its
// type allows at 32 (1000 x 768 fp32, 16 / 32 columns: 11.9 / 10.9 us).
constexpr int kApartCols = 32;
template <typename T>
__device__ __forceinline__ void norm_columns(const NormBwdArgs<T>& a, int c0, float* lds /* [waves][kApartCols] */) {
  constexpr int kRows = 4;   // whose words are on their way together
  constexpr int kLanes = kApartCols / 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, step = blockDim.x / kLanes;
  const int c = min(c0 + 8 * (lane % kLanes), a.d - 8);
  float dgamma[8], dbeta[8];
#pragma unroll
  for (int z = 0; z < 8; ++z) dgamma[z] = dbeta[z] = 0.f;
  for (int64_t first = threadIdx.x / kLanes; first < a.n_tok; first += kRows * step) {
    Raw8<T> y[kRows], dh[kRows];
    float mean[kRows], rstd[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t t = min(first + u * step, (int64_t)a.n_tok - 1);
      y[u].load(a.y + (size_t)t * a.d + c);
      dh[u].load(a.dh + (size_t)t * a.d + c);
      rstd[u] = a.rstd[t];
      mean[u] = a.layer ? a.mean[t] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      float y8[8], g8[8];
      y[u].widen(y8);
      dh[u].widen(g8);
      const bool live = first + u * step < a.n_tok;
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        dgamma[z] += live ? g8[z] * ((y8[z] - mean[u]) * rstd[u]) : 0.f;
        dbeta[z] += live ? g8[z] : 0.f;
      }
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float(&acc)[8] = which == 0 ? dgamma : dbeta;
    T* out = which == 0 ? a.dgamma : a.dbeta;
    if (!out) continue;
#pragma unroll
    for (int z = 0; z < 8; ++z)
#pragma unroll
      for (int o = kLanes; o < 64; o *= 2) acc[z] += __shfl_xor(acc[z], o, kWave);
    __syncthreads();
    if (lane < kLanes) Vec8<float>::store(lds + wave * kApartCols + lane * 8, acc);
    __syncthreads();
    if (threadIdx.x < kApartCols && c0 + (int)threadIdx.x < a.d) {
      float sum = 0.f;
      for (int w = 0; w < waves; ++w) sum += lds[w * kApartCols + threadIdx.x];
      if constexpr (sizeof(T) == 2) out[c0 + threadIdx.x].bits = (uint16_t)pack_bf16x2(sum, 0.f);
      else out[c0 + threadIdx.x] = sum;
    }
  }
}

// kGrads: 0 dx only, 1 and dgamma, 2 and dbeta.  A workgroup walks rows with the weight's gradient of its columns in
// registers; the slots of a workgroup are added through LDS, the workgroups by norm_grad_kernel, both in a fixed order.
// Memory bounds it: 8192 x 4096 bf16, rms, 43 us for three matrices read and one written (6.2 TB/s), with dropout's output 59.
// 3 (few rows): dx by the first row_wgs workgroups and the weights' gradients by workgroups of their own, which read the rows
// again, in one launch instead of two.
template <typename T, int V, int W, int kMode, int kGrads>
__global__ __launch_bounds__(64 * W * norm_max_slots(W)) void norm_bwd_kernel(NormBwdArgs<T> a) {
  constexpr int kMaxSlots = norm_max_slots(W);
  __shared__ float s_sum[2 * kMaxSlots * W * 2];
  constexpr bool kAcc = kGrads == 1 || kGrads == 2;
  __shared__ __attribute__((aligned(16))) float s_acc[kGrads == 3 ? 16 * kApartCols : kAcc && kMaxSlots > 1 ? 64 * W * V * 8 : 4];
  const int row_wgs = kGrads == 3 ? a.row_wgs : (int)gridDim.x;
  if (kGrads == 3 && (int)blockIdx.x >= row_wgs) {
    norm_columns(a, ((int)blockIdx.x - row_wgs) * kApartCols, s_acc);
    return;
  }
  const int slots = blockDim.x / (64 * W), slot = threadIdx.x / (64 * W), q = threadIdx.x % (64 * W), wave = q / 64;
  RowSum<W, kMaxSlots, 2> row_sum{s_sum};
  const uint64_t offset = kMode == kNormDrop ? drop_offset(a.drop) : 0;
  Raw8<T> gamma[V], raw_y[V], raw_dh[V], raw_dy[V];
  float dgamma[V][8], dbeta[V][8], rstd_next = 0.f, mean_next = 0.f;
  bool in[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (i * 64 * W + q) * 8;
    in[i] = c < a.d;
    gamma[i].clear();
    raw_y[i].clear();
    raw_dh[i].clear();
    raw_dy[i].clear();
    if (in[i]) gamma[i].load(a.gamma + c);
#pragma unroll
    for (int z = 0; z < 8; ++z) dgamma[i][z] = dbeta[i][z] = 0.f;
  }
  auto load = [&](int64_t t) {
    if (t >= a.n_tok) return;
    const size_t row = (size_t)t * a.d;
    rstd_next = a.rstd[t];
    if (a.layer) mean_next = a.mean[t];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * 64 * W + q) * 8;
      if (!in[i]) continue;
      raw_y[i].load(a.y + row + c);
      raw_dh[i].load(a.dh + row + c);
      if (a.dy) raw_dy[i].load(a.dy + row + c);
    }
  };
  const int64_t stride = (int64_t)row_wgs * slots;
  constexpr bool kAhead = W < 16;   // 1024 threads have 128 registers each: none for a row to come
  if (kAhead) load((int64_t)blockIdx.x * slots + slot);
  for (int64_t first = (int64_t)blockIdx.x * slots; first < a.n_tok; first += stride) {
    const int64_t t = first + slot;
    if (!kAhead) load(t);
    const bool live = t < a.n_tok;   // a slot behind the last row computes on a row of before and keeps nothing
    const size_t row = (size_t)t * a.d;
    const float rstd = rstd_next, mean = mean_next;
    // the row's values in fp32 where their words make room for the next row's, else widened again behind the sums
    constexpr int kHeld = kAhead ? V : 1;
    float g[kHeld][8], xh[kHeld][8], r[kHeld][8], s[2] = {0.f, 0.f};
    auto widen = [&](int i, float(&x8)[8], float(&g8)[8]) {
      raw_y[i].widen(x8);
      raw_dh[i].widen(g8);
#pragma unroll
      for (int z = 0; z < 8; ++z) x8[z] = in[i] ? (x8[z] - mean) * rstd : 0.f;
    };
    auto weigh = [&](int i, float(&g8)[8]) {
      float gm[8];
      gamma[i].widen(gm);
#pragma unroll
      for (int z = 0; z < 8; ++z) g8[z] *= gm[z];
    };
    auto sums = [&](int i, float(&x8)[8], float(&g8)[8]) {
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        if (kAcc) dgamma[i][z] += live ? g8[z] * x8[z] : 0.f;
        if (kGrads == 2) dbeta[i][z] += live ? g8[z] : 0.f;
      }
      weigh(i, g8);
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        s[0] += g8[z];
        s[1] += g8[z] * x8[z];
      }
    };
    if constexpr (kAhead) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        widen(i, xh[i], g[i]);
        raw_dy[i].widen(r[i]);
      }
      load(t + stride);
#pragma unroll
      for (int i = 0; i < V; ++i) sums(i, xh[i], g[i]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        widen(i, xh[0], g[0]);
        sums(i, xh[0], g[0]);
        raw_y[i].forget();
        raw_dh[i].forget();
        raw_dy[i].forget();
        gamma[i].forget();
      }
    }
    row_sum(s, slot, wave);
    const float m0 = a.layer ? s[0] * a.inv_d : 0.f, m1 = s[1] * a.inv_d;
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (!in[i]) continue;
      constexpr bool held = kAhead;
      const int c = (i * 64 * W + q) * 8, k = held ? i : 0;
      if (!held) {
        widen(i, xh[k], g[k]);
        weigh(i, g[k]);
        raw_dy[i].widen(r[k]);
      }
#pragma unroll
      for (int z = 0; z < 8; ++z) g[k][z] = rstd * (g[k][z] - m0 - xh[k][z] * m1) + r[k][z];
      store8(a.dx + row + c, g[k], kMode == kNormPlain && a.past);
      if (kMode != kNormPlain) {
        if (kMode == kNormDrop) drop8(a.drop, offset, (uint32_t)t, c / 8, g[k]);
        Vec8<T>::store(a.dout + row + c, g[k]);
      }
    }
  }
  if constexpr (kAcc) {
    float* p = a.part + (size_t)blockIdx.x * 2 * a.d;
#pragma unroll
    for (int which = 0; which < kGrads; ++which) {
      float(&acc)[V][8] = which == 0 ? dgamma : dbeta;
      if constexpr (kMaxSlots > 1) {
        for (int other = 1; other < slots; ++other) {
          __syncthreads();
          if (slot == other)
#pragma unroll
            for (int i = 0; i < V; ++i) Vec8<float>::store(s_acc + (i * 64 * W + q) * 8, acc[i]);
          __syncthreads();
          if (slot == 0)
#pragma unroll
            for (int i = 0; i < V; ++i) {
              float r[8];
              Vec8<float>::load(s_acc + (i * 64 * W + q) * 8, r);
#pragma unroll
              for (int z = 0; z < 8; ++z) acc[i][z] += r[z];
            }
        }
      }
      if (slot == 0)
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (in[i]) Vec8<float>::store(p + (size_t)which * a.d + (i * 64 * W + q) * 8, acc[i]);
    }
  }
}

// dgamma and dbeta (blockIdx.y) from the workgroups' partial sums: 8 threads along 32 columns, 64 along the workgroups.  Bound by
// one or two round trips to memory: 5.1 us for 512 workgroups of 4096 columns (16 columns a workgroup 5.7; a loop over the
// workgroups that does not ask ahead 8 to 10).
template <typename T>
__global__ __launch_bounds__(512) void norm_grad_kernel(const float* __restrict__ part, int n_part, int d, T* dgamma, T* dbeta) {
  __shared__ __attribute__((aligned(16))) float s[64][32];
  const int q = threadIdx.x & 7, g = threadIdx.x >> 3, c = blockIdx.x * 32 + q * 4;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (c < d && g < n_part)
    v = sum_places(reinterpret_cast<const f32x4*>(part + ((size_t)g * 2 + blockIdx.y) * d + c), (n_part - g + 63) / 64, (size_t)32 * d);
  *reinterpret_cast<f32x4*>(&s[g][q * 4]) = v;
  __syncthreads();
  if (threadIdx.x < 256) {   // eight threads a column
    const int lc = threadIdx.x >> 3, k = threadIdx.x & 7, col = blockIdx.x * 32 + lc;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += s[k * 8 + i][lc];
#pragma unroll
    for (int o = 1; o < 8; o *= 2) sum += __shfl_xor(sum, o, kWave);
    if (k == 0 && col < d) {
      T* out = blockIdx.y == 0 ? dgamma : dbeta;
      if constexpr (sizeof(T) == 2) out[col].bits = (uint16_t)pack_bf16x2(sum, 0.f);
      else out[col] = sum;
    }
  }
}

}  // namespace meft
