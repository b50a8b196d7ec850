// The router's gradient: from the gradient of its scores p[t, b] = Wg[b, :] . h[t, :] + bias[b]
//
//   dh[t, :] = add[t, :] + sum_b ds[t, b] Wg[b, :]      dWg[b, :] = sum_t ds[t, b] h[t, :]      dbias[b] = sum_t ds[t, b]
//
// Both contractions are far below the matrix cores' rate at the number of blocks in use (4 T d B flop against 6 T d bytes at
// bf16): reading h and add and writing dh bounds them.  So neither uses LDS for operands: a wave loads four consecutive columns
// of eight rows per lane straight into registers, where swapping halves of words gives the matrix instruction's operand
// (it wants eight rows of one column per lane); lane l then holds columns 4 (l % 32) + j of its four result tiles j, so that a
// result row leaves as one 8- or 16-byte word per lane, 32 lanes on consecutive addresses.
//
// ds arrives in fp32.  bf16 shapes split it in two bf16 parts, high and low, and multiply both: rounded to one, its error would
// be as large as that of rounding the result; the matrix cores have the time.  fp32 shapes use fp32 matrix instructions.
#pragma once
#include "common.h"

namespace meft {

typedef u32x2 u32x2_8 __attribute__((aligned(8)));

// eight rows of four columns, and the operands that they give
template <typename T>
struct Rows8;

template <>
struct Rows8<bf16_t> {
  u32x2 w[8];
  __device__ __forceinline__ void load(int u, const bf16_t* p) { w[u] = *reinterpret_cast<const u32x2*>(p); }
  // the eight rows of column j
  __device__ __forceinline__ bf16x8 operand(int j) const {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r[i] = __builtin_amdgcn_perm(w[2 * i + 1][j / 2], w[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
    return __builtin_bit_cast(bf16x8, r);
  }
};

template <>
struct Rows8<float> {
  f32x4 w[8];
  __device__ __forceinline__ void load(int u, const float* p) { w[u] = *reinterpret_cast<const f32x4*>(p); }
};

// acc[j] += a (8 values of a row of the left operand per lane) * rows, for the four columns j
__device__ __forceinline__ void mma_rows8(const float (&a)[8], const Rows8<bf16_t>& rows, f32x16 (&acc)[4]) {
  u32x4 hi, lo;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    hi[i] = pack_bf16x2(a[2 * i], a[2 * i + 1]);
    lo[i] = pack_bf16x2(a[2 * i] - __uint_as_float(hi[i] << 16), a[2 * i + 1] - __uint_as_float(hi[i] & 0xFFFF0000u));
  }
  const bf16x8 h8 = __builtin_bit_cast(bf16x8, hi), l8 = __builtin_bit_cast(bf16x8, lo);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bf16x8 b = rows.operand(j);
    acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(h8, b, acc[j], 0, 0, 0);
    acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(l8, b, acc[j], 0, 0, 0);
  }
}
__device__ __forceinline__ void mma_rows8(const float (&a)[8], const Rows8<float>& rows, f32x16 (&acc)[4]) {
#pragma unroll
  for (int u = 0; u < 8; ++u)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[u], rows.w[u][j], acc[j], 0, 0, 0);
}

// row of a 32 x 32 result that register r of this lane holds
__device__ __forceinline__ int tile_row(int r, int lane) { return 8 * (r / 4) + 4 * (lane / 32) + r % 4; }

constexpr int kRgCols = 128;    // columns of a wave's tile
constexpr int kRgTok = 64;      // dh: tokens of a wave's tile

template <typename T>
struct RouteGradArgs {
  const T *h, *Wg, *add;
  const float* ds;
  T *dh, *dWg;
  float *dbias, *part, *part_bias;   // part: [split][B][d], where there is more than one split
  int n_tok, d, B;
  int slices;                        // ceil(d / kRgCols)
  int m_waves, splits, per_split;    // dWg: waves along the blocks, splits of the tokens, tokens of a split (a multiple of 16)
};

template <typename T>
__device__ __forceinline__ void store4(T* p, const float (&v)[4]) {
  if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
}
template <typename T>
__device__ __forceinline__ void load4(const T* p, float (&v)[4]) {
  if constexpr (sizeof(T) == 2) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
    v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xFFFF0000u);
    v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xFFFF0000u);
  } else {
    const f32x4 w = *reinterpret_cast<const f32x4*>(p);
    v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
  }
}

// dh.  A wave: 64 tokens x 128 columns; the four waves of a workgroup take consecutive tokens of the same columns, whose
// router rows they then find in the vector cache.  Grid: slices * ceil(T / 256), the slices fastest.
template <typename T>
__global__ __launch_bounds__(256) void route_dh_kernel(RouteGradArgs<T> a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int tile = blockIdx.x / a.slices, slice = blockIdx.x - tile * a.slices;
  const int64_t t0 = (int64_t)tile * 4 * kRgTok + wave * kRgTok;
  if (t0 >= a.n_tok) return;
  const int c = slice * kRgCols + 4 * (lane & 31), cc = min(c, a.d - 4);
  const float* ds[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) ds[m] = a.ds + (size_t)min(t0 + m * 32 + (lane & 31), (int64_t)a.n_tok - 1) * a.B;
  f32x16 acc[2][4];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[m][j][r] = 0.f;
  int b0 = 0;
  for (; b0 + 16 <= a.B; b0 += 16) {
    const int b = b0 + 8 * half;
    Rows8<T> rows;
#pragma unroll
    for (int u = 0; u < 8; ++u) rows.load(u, a.Wg + (size_t)(b + u) * a.d + cc);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float x[8];
      *reinterpret_cast<u32x4*>(x) = *reinterpret_cast<const u32x4_dw*>(ds[m] + b);
      *reinterpret_cast<u32x4*>(x + 4) = *reinterpret_cast<const u32x4_dw*>(ds[m] + b + 4);
      mma_rows8(x, rows, acc[m]);
    }
  }
  if (b0 < a.B) {
    const int b = b0 + 8 * half;
    Rows8<T> rows;
#pragma unroll
    for (int u = 0; u < 8; ++u) rows.load(u, a.Wg + (size_t)min(b + u, a.B - 1) * a.d + cc);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float v = ds[m][min(b + u, a.B - 1)];
        x[u] = b + u < a.B ? v : 0.f;
      }
      mma_rows8(x, rows, acc[m]);
    }
  }
  if (c >= a.d) return;
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int64_t t = t0 + m * 32 + tile_row(r, lane);
      if (t >= a.n_tok) continue;
      float v[4] = {acc[m][0][r], acc[m][1][r], acc[m][2][r], acc[m][3][r]};
      if (a.add) {
        float x[4];
        load4(a.add + (size_t)t * a.d + c, x);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += x[j];
      }
      store4(a.dh + (size_t)t * a.d + c, v);
    }
}

// dWg and dbias.  A wave: 32 M blocks x 128 columns over a share of the tokens, 16 at a time; a_waves waves lie along the
// blocks, the others share out the tokens and are added through LDS.  Grid: (slices, ceil(B / (32 M m_waves)), splits).
template <typename T, int M>
__global__ __launch_bounds__(256) void route_dw_kernel(RouteGradArgs<T> a) {
  __shared__ float s_acc[2][M * 64][64];
  __shared__ float s_bias[4][M][32];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int m_waves = a.m_waves, k_waves = 4 / m_waves, mw = wave % m_waves, kw = wave / m_waves;
  const int b0 = ((int)blockIdx.y * m_waves + mw) * 32 * M;
  const int c = blockIdx.x * kRgCols + 4 * (lane & 31), cc = min(c, a.d - 4);
  const int64_t begin = (int64_t)blockIdx.z * a.per_split, end = min(begin + a.per_split, (int64_t)a.n_tok);
  int bb[M];
#pragma unroll
  for (int m = 0; m < M; ++m) bb[m] = min(b0 + 32 * m + (lane & 31), a.B - 1);
  f32x16 acc[M][4];
  float bias[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    bias[m] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[m][j][r] = 0.f;
  }
  for (int64_t t0 = begin + 16 * kw; t0 < end; t0 += 16 * k_waves) {
    const int64_t t = t0 + 8 * half;
    Rows8<T> rows;
    float x[M][8];
    const bool whole = t0 + 16 <= end;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t tt = whole ? t + u : min(t + u, end - 1);
      rows.load(u, a.h + (size_t)tt * a.d + cc);
#pragma unroll
      for (int m = 0; m < M; ++m) x[m][u] = a.ds[(size_t)tt * a.B + bb[m]];
    }
    if (!whole) {
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int m = 0; m < M; ++m) x[m][u] = t + u < end ? x[m][u] : 0.f;
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
      mma_rows8(x[m], rows, acc[m]);
      if (blockIdx.x == 0) bias[m] += ((x[m][0] + x[m][1]) + (x[m][2] + x[m][3])) + ((x[m][4] + x[m][5]) + (x[m][6] + x[m][7]));
    }
  }
  // the waves that shared out the tokens, in pairs
  for (int n = k_waves / 2; n > 0; n /= 2) {
    __syncthreads();
    float(*s)[64] = s_acc[(kw % n) * m_waves + mw];
    if (kw >= n && kw < 2 * n) {
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[(m * 4 + j) * 16 + r][lane] = acc[m][j][r];
    }
    __syncthreads();
    if (kw < n) {
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[m][j][r] += s[(m * 4 + j) * 16 + r][lane];
    }
  }
  if (blockIdx.x == 0) {
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const float v = bias[m] + __shfl_xor(bias[m], 32, kWave);
      if (half == 0) s_bias[wave][m][lane] = v;
    }
    __syncthreads();
    if (kw == 0 && half == 0 && a.dbias) {
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const int b = b0 + 32 * m + lane;
        float v = 0.f;
        for (int k = 0; k < k_waves; ++k) v += s_bias[k * m_waves + mw][m][lane];
        if (b < a.B) (a.splits > 1 ? a.part_bias + (size_t)blockIdx.z * a.B : a.dbias)[b] = v;
      }
    }
  }
  if (kw != 0 || c >= a.d || !a.dWg) return;
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int b = b0 + 32 * m + tile_row(r, lane);
      if (b >= a.B) continue;
      const float v[4] = {acc[m][0][r], acc[m][1][r], acc[m][2][r], acc[m][3][r]};
      if (a.splits > 1) store4(a.part + ((size_t)blockIdx.z * a.B + b) * a.d + c, v);
      else store4(a.dWg + (size_t)b * a.d + c, v);
    }
}

// the splits of dWg and dbias added up, in order; one workgroup more than dWg's quadruples need writes dbias
template <typename T>
__global__ __launch_bounds__(256) void route_dw_join_kernel(RouteGradArgs<T> a) {
  const int64_t n = (int64_t)a.B * a.d, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (a.dbias && blockIdx.x == gridDim.x - 1)
    for (int b = threadIdx.x; b < a.B; b += 256) {
      float v = 0.f;
      for (int s = 0; s < a.splits; ++s) v += a.part_bias[(size_t)s * a.B + b];
      a.dbias[b] = v;
    }
  if (i >= n || !a.dWg) return;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.splits; ++s) {
    float x[4];
    load4(a.part + (size_t)s * n + i, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += x[j];
  }
  store4(a.dWg + i, v);
}

}  // namespace meft
