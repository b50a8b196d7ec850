// The router's balance loss, its counts and its gradient.  For the n valid tokens, B blocks, e of them per token:
//
//   P[t, .] = softmax(scores[t, .]),  lse_t = log sum exp scores[t, .]
//   f_b = counts_b / (n e),  L = B sum_b f_b (1/n) sum_t P[t, b],  Z = (1/n) sum_t lse_t^2,  loss = balance L + z Z
//   dscores[t, b] = dloss P[t, b] ((balance B / n) (f_b - sum_b' f_b' P[t, b']) + (2 z / n) lse_t)
//
// The counts carry no gradient (a selection has none).  A row of scores that are all -inf counts as a token that is not
// valid: it has no softmax.
//
// W waves hold a row in registers, Z scores per lane; W = 1 up to 1024 blocks.
#pragma once
#include "common.h"

namespace meft {

__device__ __forceinline__ float wave_max_f32(float v) {
#define MEFT_DPP_FMAX(ctrl) \
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp((int)__float_as_uint(v), (int)__float_as_uint(v), ctrl, 0xF, 0xF, false)))
  MEFT_DPP_FMAX(0xB1);
  MEFT_DPP_FMAX(0x4E);
  MEFT_DPP_FMAX(0x141);
  MEFT_DPP_FMAX(0x140);
#undef MEFT_DPP_FMAX
  v = fmaxf(v, __shfl_xor(v, 16, kWave));
  return fmaxf(v, __shfl_xor(v, 32, kWave));
}

// sum over the row's waves of a value that is the same in every lane of a wave; two barriers
template <int W, typename F>
__device__ __forceinline__ float row_join(float v, float* lds, F&& join) {
  if constexpr (W > 1) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < W; ++w) v = join(v, lds[w]);
  }
  return v;
}

// x[z] becomes the probability; returns whether the row has any score above -inf.  NaN stays NaN.
template <int Z, int W>
__device__ __forceinline__ bool row_softmax(const float* row, int B, int lane0, float* lds, float (&x)[Z], float& lse) {
  float top = -__builtin_inff();
  bool any = false;
#pragma unroll
  for (int z = 0; z < Z; ++z) {
    const int b = z * 64 * W + lane0;
    x[z] = b < B ? row[b] : -__builtin_inff();
    any |= x[z] != -__builtin_inff();
    top = fmaxf(top, x[z]);
  }
  top = row_join<W>(wave_max_f32(top), lds, [](float a, float b) { return fmaxf(a, b); });
  const float live = row_join<W>(__ballot(any) ? 1.f : 0.f, lds, [](float a, float b) { return a + b; });
  if (live == 0.f) return false;
  float sum = 0.f;
#pragma unroll
  for (int z = 0; z < Z; ++z) {
    x[z] = z * 64 * W + lane0 < B ? expf(x[z] - top) : 0.f;
    sum += x[z];
  }
  sum = row_join<W>(wave_sum(sum), lds, [](float a, float b) { return a + b; });
  lse = top + logf(sum);
  const float inv = 1.f / sum;
#pragma unroll
  for (int z = 0; z < Z; ++z) x[z] *= inv;
  return true;
}

struct BalancePart {
  float* prob;       // [workgroup][B]
  int32_t* count;    // [workgroup][B]
  float* lse2;       // [workgroup]
  int32_t* tokens;   // [workgroup]
  float* dot;        // [workgroup of the second launch]
  uint32_t* ticket;
};

// LDS: counts [B] ints, then for W == 1 the waves' probabilities [4][B]
template <int Z, int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void balance_part_kernel(const float* __restrict__ scores,
                                                                             const int32_t* __restrict__ block_idx,
                                                                             const uint8_t* __restrict__ valid, int n_tok, int B,
                                                                             int e, BalancePart part) {
  extern __shared__ int32_t s_cnt[];
  __shared__ float s_join[16], s_lse2[4];
  __shared__ int32_t s_tok[4];
  constexpr int kThreads = W == 1 ? 256 : 64 * W, kRows = W == 1 ? 4 : 1;
  const int tid = threadIdx.x, wave = tid / 64, lane0 = W == 1 ? (tid & 63) : tid, slot = W == 1 ? wave : 0;
  for (int b = tid; b < B; b += kThreads) s_cnt[b] = 0;
  if (blockIdx.x == 0 && tid == 0) *part.ticket = 0u;   // of the next launch
  __syncthreads();
  float acc[Z], lse2 = 0.f;
  int n = 0;
#pragma unroll
  for (int z = 0; z < Z; ++z) acc[z] = 0.f;
  for (int64_t t = (int64_t)blockIdx.x * kRows + slot; t < n_tok; t += (int64_t)gridDim.x * kRows) {
    if (valid && !valid[t]) continue;
    float x[Z], lse;
    if (!row_softmax<Z, W>(scores + (size_t)t * B, B, lane0, s_join, x, lse)) continue;
#pragma unroll
    for (int z = 0; z < Z; ++z) acc[z] += x[z];
    lse2 += lse * lse;
    ++n;
    for (int q = lane0; q < e; q += 64 * W) {
      const int b = block_idx[(size_t)t * e + q];
      if ((unsigned)b < (unsigned)B) atomicAdd(&s_cnt[b], 1);
    }
  }
  float* s_prob = reinterpret_cast<float*>(s_cnt + B);
  if constexpr (W == 1) {
#pragma unroll
    for (int z = 0; z < Z; ++z)
      if (z * 64 + lane0 < B) s_prob[wave * B + z * 64 + lane0] = acc[z];
    if (lane0 == 0) { s_lse2[wave] = lse2; s_tok[wave] = n; }
  }
  __syncthreads();
  float* prob = part.prob + (size_t)blockIdx.x * B;
  int32_t* count = part.count + (size_t)blockIdx.x * B;
  if constexpr (W == 1) {
    for (int b = tid; b < B; b += kThreads) prob[b] = (s_prob[b] + s_prob[B + b]) + (s_prob[2 * B + b] + s_prob[3 * B + b]);
    if (tid == 0) { lse2 = (s_lse2[0] + s_lse2[1]) + (s_lse2[2] + s_lse2[3]); n = s_tok[0] + s_tok[1] + s_tok[2] + s_tok[3]; }
  } else {
#pragma unroll
    for (int z = 0; z < Z; ++z)
      if (z * 64 * W + lane0 < B) prob[z * 64 * W + lane0] = acc[z];
  }
  for (int b = tid; b < B; b += kThreads) count[b] = s_cnt[b];
  if (tid == 0) { part.lse2[blockIdx.x] = lse2; part.tokens[blockIdx.x] = n; }
}

// Joins the workgroups' partial sums, 64 blocks and 16 groups of workgroups per workgroup of 1024 threads; the workgroup
// that is done last adds the others' shares of the loss up in order.
__global__ __launch_bounds__(1024) void balance_join_kernel(BalancePart part, int n_part, int B, int e, float balance, float z,
                                                            int32_t* __restrict__ counts, int32_t* __restrict__ n_valid,
                                                            float* __restrict__ prob, float* __restrict__ loss) {
  __shared__ float s_prob[16][64], s_lse2[16];
  __shared__ int32_t s_cnt[16][64], s_tok[16];
  __shared__ uint32_t s_last;
  const int tid = threadIdx.x, lane = tid & 63, g = tid >> 6, b = blockIdx.x * 64 + lane;
  float p = 0.f;
  int32_t c = 0;
  if (b < B)
    for (int i = g; i < n_part; i += 16) {
      p += part.prob[(size_t)i * B + b];
      c += part.count[(size_t)i * B + b];
    }
  s_prob[g][lane] = p;
  s_cnt[g][lane] = c;
  __syncthreads();
  if (g == 0) {
    p = 0.f;
    c = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) { p += s_prob[i][lane]; c += s_cnt[i][lane]; }
    if (b < B) { prob[b] = p; counts[b] = c; }
    const float dot = wave_sum(p * (float)c);
    if (lane == 0) {
      __hip_atomic_store(&part.dot[blockIdx.x], dot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      s_last = __hip_atomic_fetch_add(part.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
  }
  __syncthreads();
  if (!s_last) return;
  float l2 = 0.f;
  int32_t n = 0;
  for (int i = tid; i < n_part; i += 1024) { l2 += part.lse2[i]; n += part.tokens[i]; }
  l2 = wave_sum(l2);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, kWave);
  if (lane == 0) { s_lse2[g] = l2; s_tok[g] = n; }
  __syncthreads();
  if (tid == 0) {
    l2 = 0.f;
    n = 0;
    for (int i = 0; i < 16; ++i) { l2 += s_lse2[i]; n += s_tok[i]; }
    float dot = 0.f;
    for (unsigned i = 0; i < gridDim.x; ++i) dot += __hip_atomic_load(&part.dot[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const float inv = n > 0 ? 1.f / (float)n : 0.f;
    const float lb = (float)B / (float)e * dot * inv * inv, lz = l2 * inv;
    *n_valid = n;
    // a term of weight 0 is left out, so that an overflow of the other's does not reach the sum
    loss[0] = (balance != 0.f ? balance * lb : 0.f) + (z != 0.f ? z * lz : 0.f);
    loss[1] = lb;
    loss[2] = lz;
  }
}

template <int Z, int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void balance_grad_kernel(const float* scores,
                                                                             const int32_t* __restrict__ counts,
                                                                             const int32_t* __restrict__ n_valid,
                                                                             const uint8_t* __restrict__ valid,
                                                                             const float* __restrict__ dloss, int n_tok, int B,
                                                                             int e, float balance, float z_weight,
                                                                             float* dscores) {
  __shared__ float s_join[16];
  constexpr int kRows = W == 1 ? 4 : 1;
  const int tid = threadIdx.x, lane0 = W == 1 ? (tid & 63) : tid, slot = W == 1 ? tid / 64 : 0;
  const int n = *n_valid;
  const float inv = n > 0 ? 1.f / (float)n : 0.f, g = dloss ? *dloss : 1.f;
  const float cb = g * balance * (float)B * inv, cz = g * z_weight * 2.f * inv;
  float f[Z];
#pragma unroll
  for (int z = 0; z < Z; ++z) {
    const int b = z * 64 * W + lane0;
    f[z] = b < B ? (float)counts[b] * (inv / (float)e) : 0.f;
  }
  for (int64_t t = (int64_t)blockIdx.x * kRows + slot; t < n_tok; t += (int64_t)gridDim.x * kRows) {
    float* o = dscores + (size_t)t * B;
    float x[Z], lse;
    const bool live = (!valid || valid[t]) && row_softmax<Z, W>(scores + (size_t)t * B, B, lane0, s_join, x, lse);
    float mean = 0.f;
    if (live) {
#pragma unroll
      for (int z = 0; z < Z; ++z) mean += f[z] * x[z];
      mean = row_join<W>(wave_sum(mean), s_join, [](float a, float b) { return a + b; });
    }
    const float lz = cz != 0.f && live ? cz * lse : 0.f;
#pragma unroll
    for (int z = 0; z < Z; ++z)
      if (z * 64 * W + lane0 < B) o[z * 64 * W + lane0] = live ? x[z] * (cb * (f[z] - mean) + lz) : 0.f;
  }
}

}  // namespace meft
