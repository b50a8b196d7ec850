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

template <typename T>
struct Raw8 {
  u32x4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) w[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) w[i] = u32x4{0u, 0u, 0u, 0u};
  }
  __device__ __forceinline__ void widen(float (&v)[8]) const {
    if constexpr (sizeof(T) == 2) {
      Vec8<bf16_t>::widen(w[0], v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i / 4][i % 4]);
    }
  }
};

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
template <int W, int kSlots, int kValues>
struct RowSum {
  float* lds;   // [2][kSlots][W][kValues]
  int turn = 0;
  __device__ __forceinline__ void operator()(float (&v)[kValues], int slot, int wave) {
#pragma unroll
    for (int i = 0; i < kValues; ++i) v[i] = wave_sum(v[i]);
    if constexpr (W > 1) {
      float* p = lds + (size_t)((turn * kSlots + slot) * W) * kValues;
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
  DropArgs drop;
};

template <typename T, int V, int W, int kMode>
__global__ __launch_bounds__(W > 4 ? 64 * W : 256) void norm_fwd_kernel(NormFwdArgs<T> a) {
  constexpr int kSlots = W > 4 ? 1 : 4 / W;
  __shared__ float s_sum[2 * kSlots * W];
  const int slot = threadIdx.x / (64 * W), q = threadIdx.x % (64 * W), wave = q / 64;
  RowSum<W, kSlots, 1> row_sum{s_sum};
  const uint64_t offset = kMode == kNormDrop ? drop_offset(a.drop) : 0;
  Raw8<T> gamma[V], beta[V];
  bool in[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (i * 64 * W + q) * 8;
    in[i] = c < a.d;
    gamma[i].clear();
    beta[i].clear();
    if (in[i]) gamma[i].load(a.gamma + c);
    if (in[i] && a.beta) beta[i].load(a.beta + c);
  }
  for (int64_t first = (int64_t)blockIdx.x * kSlots; first < a.n_tok; first += (int64_t)gridDim.x * kSlots) {
    const int64_t t = first + slot;
    const bool live = t < a.n_tok;
    const size_t row = (size_t)t * a.d;
    float v[V][8];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * 64 * W + q) * 8;
#pragma unroll
      for (int z = 0; z < 8; ++z) v[i][z] = 0.f;
      if (!live || !in[i]) continue;
      Vec8<T>::load(a.x + row + c, v[i]);
      if (kMode != kNormPlain) {
        float o[8];
        Vec8<T>::load(a.out + row + c, o);
        if (kMode == kNormDrop) drop8(a.drop, offset, (uint32_t)t, c / 8, o);
#pragma unroll
        for (int z = 0; z < 8; ++z) v[i][z] += o[z];
        round8<T>(v[i]);   // the norm is of the stream as it is stored, which is what the backward reads
        Vec8<T>::store(a.y + row + c, v[i]);
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
      Vec8<T>::store(a.h + row + (i * 64 * W + q) * 8, v[i]);
    }
  }
}

template <typename T>
struct NormBwdArgs {
  const T *y, *gamma, *dh, *dy;
  const float *mean, *rstd;
  T *dx, *dout;
  float* part;   // [workgroup][dgamma, dbeta][d]
  int n_tok, d, layer;
  float inv_d;
  DropArgs drop;
};

// kGrads: 0 dx only, 1 and dgamma, 2 and dbeta.  A workgroup walks rows with the weight's gradient of its columns in
// registers; the slots of a workgroup are added through LDS, the workgroups by norm_grad_kernel, both in a fixed order.
template <typename T, int V, int W, int kMode, int kGrads>
__global__ __launch_bounds__(W > 8 ? 64 * W : 512) void norm_bwd_kernel(NormBwdArgs<T> a) {
  constexpr int kSlots = W > 8 ? 1 : 8 / W;
  __shared__ float s_sum[2 * kSlots * W * 2];
  __shared__ __attribute__((aligned(16))) float s_acc[kGrads && kSlots > 1 ? 64 * W * V * 8 : 4];
  const int slot = threadIdx.x / (64 * W), q = threadIdx.x % (64 * W), wave = q / 64;
  RowSum<W, kSlots, 2> row_sum{s_sum};
  const uint64_t offset = kMode == kNormDrop ? drop_offset(a.drop) : 0;
  Raw8<T> gamma[V];
  float dgamma[V][8], dbeta[V][8];
  bool in[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (i * 64 * W + q) * 8;
    in[i] = c < a.d;
    gamma[i].clear();
    if (in[i]) gamma[i].load(a.gamma + c);
#pragma unroll
    for (int z = 0; z < 8; ++z) dgamma[i][z] = dbeta[i][z] = 0.f;
  }
  for (int64_t first = (int64_t)blockIdx.x * kSlots; first < a.n_tok; first += (int64_t)gridDim.x * kSlots) {
    const int64_t t = first + slot;
    const bool live = t < a.n_tok;
    const size_t row = (size_t)t * a.d;
    const float rstd = live ? a.rstd[t] : 0.f, mean = live && a.layer ? a.mean[t] : 0.f;
    float g[V][8], xh[V][8], s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * 64 * W + q) * 8;
#pragma unroll
      for (int z = 0; z < 8; ++z) g[i][z] = xh[i][z] = 0.f;
      if (!live || !in[i]) continue;
      Vec8<T>::load(a.y + row + c, xh[i]);
      Vec8<T>::load(a.dh + row + c, g[i]);
      float gm[8];
      gamma[i].widen(gm);
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        xh[i][z] = (xh[i][z] - mean) * rstd;
        if (kGrads > 0) dgamma[i][z] += g[i][z] * xh[i][z];
        if (kGrads > 1) dbeta[i][z] += g[i][z];
        g[i][z] *= gm[z];
        s[0] += g[i][z];
        s[1] += g[i][z] * xh[i][z];
      }
    }
    row_sum(s, slot, wave);
    const float m0 = a.layer ? s[0] * a.inv_d : 0.f, m1 = s[1] * a.inv_d;
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (!in[i]) continue;
      const int c = (i * 64 * W + q) * 8;
      float r[8];
#pragma unroll
      for (int z = 0; z < 8; ++z) g[i][z] = rstd * (g[i][z] - m0 - xh[i][z] * m1);
      if (a.dy) {
        Vec8<T>::load(a.dy + row + c, r);
#pragma unroll
        for (int z = 0; z < 8; ++z) g[i][z] += r[z];
      }
      Vec8<T>::store(a.dx + row + c, g[i]);
      if (kMode != kNormPlain) {
        if (kMode == kNormDrop) drop8(a.drop, offset, (uint32_t)t, c / 8, g[i]);
        Vec8<T>::store(a.dout + row + c, g[i]);
      }
    }
  }
  if constexpr (kGrads > 0) {
    float* p = a.part + (size_t)blockIdx.x * 2 * a.d;
#pragma unroll
    for (int which = 0; which < kGrads; ++which) {
      float(&acc)[V][8] = which == 0 ? dgamma : dbeta;
      if constexpr (kSlots > 1) {
        for (int other = 1; other < kSlots; ++other) {
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

// dgamma and dbeta (blockIdx.y) from the workgroups' partial sums: 16 threads along 64 columns, 16 along the workgroups
template <typename T>
__global__ __launch_bounds__(256) void norm_grad_kernel(const float* __restrict__ part, int n_part, int d, T* dgamma, T* dbeta) {
  __shared__ __attribute__((aligned(16))) float s[16][64];
  const int q = threadIdx.x & 15, g = threadIdx.x >> 4, c = blockIdx.x * 64 + q * 4;
  const float* p = part + (size_t)blockIdx.y * d;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (c < d)
    for (int i = g; i < n_part; i += 16) v += *reinterpret_cast<const f32x4*>(p + (size_t)i * 2 * d + c);
  *reinterpret_cast<f32x4*>(&s[g][q * 4]) = v;
  __syncthreads();
  const int col = blockIdx.x * 64 + threadIdx.x;
  if (threadIdx.x < 64 && col < d) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += s[i][threadIdx.x];
    T* o = blockIdx.y == 0 ? dgamma : dbeta;
    if constexpr (sizeof(T) == 2) o[col].bits = (uint16_t)pack_bf16x2(sum, 0.f);
    else o[col] = sum;
  }
}

}  // namespace meft
