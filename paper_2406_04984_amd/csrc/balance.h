// The router's balance loss, its counts and its gradient.  For the n valid tokens, B blocks, e of them per token:
//
//   P[t, .] = softmax(scores[t, .]),  lse_t = log sum exp scores[t, .]
//   f_b = counts_b / (n e),  L = B sum_b f_b (1/n) sum_t P[t, b],  Z = (1/n) sum_t lse_t^2,  loss = balance L + z Z
//   dscores[t, b] = dloss P[t, b] ((balance B / n) (f_b - sum_b' f_b' P[t, b']) + (2 z / n) lse_t)
//
// The counts carry no gradient (a selection has none).  A row of scores that are all -inf counts as a token that is not
// valid: it has no softmax.
//
// W waves hold a row in registers, Z scores per lane; W = 1 up to 1024 blocks.  16384 x 256: partial sums 7.5 us, their join
// 5.5, the gradient 10.1 (17, 0.5 and 34 MB); 2048 x 64: 3.9, 3.3, 3.2.  Neither memory (5.2 TB/s would be 3.2 and 6.5 us) nor the
// vector instructions alone bound the large ones: by the counters a row takes 135 and 171 of these, which keep the vector units busy
// for 3.8 and 4.8 us, and the waves spend 60 % of their time waiting, with one row each asked for ahead.  For few rows it is the
// launches.
#pragma once
#include "common.h"

namespace meft {

// Sum and maximum over a wave, the same in all lanes, by moves inside the vector unit alone: a permute through LDS takes longer
// than all else that a row needs.
__device__ __forceinline__ float wave_total(float v) {
#define MEFT_DPP_ADDF(ctrl, rows) v += __builtin_amdgcn_update_dpp(0.f, v, ctrl, rows, 0xF, false)
  MEFT_DPP_ADDF(0xB1, 0xF);    // quad_perm [1,0,3,2]
  MEFT_DPP_ADDF(0x4E, 0xF);    // quad_perm [2,3,0,1]
  MEFT_DPP_ADDF(0x141, 0xF);   // row_half_mirror
  MEFT_DPP_ADDF(0x140, 0xF);   // row_mirror: every lane holds its row's sum
  MEFT_DPP_ADDF(0x142, 0xA);   // row_bcast:15 into rows 1 and 3
  MEFT_DPP_ADDF(0x143, 0xC);   // row_bcast:31 into rows 2 and 3: row 3 holds the wave's
#undef MEFT_DPP_ADDF
  return __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}
__device__ __forceinline__ float wave_top(float v) {
#define MEFT_DPP_MAXF(ctrl, rows) \
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp((int)__float_as_uint(v), (int)__float_as_uint(v), ctrl, rows, 0xF, false)))
  MEFT_DPP_MAXF(0xB1, 0xF);
  MEFT_DPP_MAXF(0x4E, 0xF);
  MEFT_DPP_MAXF(0x141, 0xF);
  MEFT_DPP_MAXF(0x140, 0xF);
  MEFT_DPP_MAXF(0x142, 0xA);
  MEFT_DPP_MAXF(0x143, 0xC);
#undef MEFT_DPP_MAXF
  return __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// joins the waves' values of a row, each the same in all lanes of its wave; two barriers
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

// Z scores per lane: quads of consecutive ones where Z allows it, so that a row comes in 16-byte words
template <int Z, int W>
struct RowMap {
  static constexpr int kQuad = Z % 4 == 0 ? 4 : 1;
  // block of a lane's z-th score
  static __device__ __forceinline__ int block(int z, int lane0) { return (z / kQuad) * 64 * W * kQuad + lane0 * kQuad + z % kQuad; }
  static __device__ __forceinline__ void load(const float* row, int B, int lane0, float (&x)[Z]) {
#pragma unroll
    for (int z = 0; z < Z; z += kQuad) {
      const int b = block(z, lane0);
      if (kQuad == 4 && B % 4 == 0) {
        f32x4 v = f32x4{1.f, 1.f, 1.f, 1.f} * -__builtin_inff();
        if (b < B) v = *reinterpret_cast<const f32x4*>(row + b);
#pragma unroll
        for (int i = 0; i < kQuad; ++i) x[z + i] = v[i];
      } else {
#pragma unroll
        for (int i = 0; i < kQuad; ++i) x[z + i] = b + i < B ? row[b + i] : -__builtin_inff();
      }
    }
  }
  static __device__ __forceinline__ void store(float* row, int B, int lane0, const float (&x)[Z]) {
#pragma unroll
    for (int z = 0; z < Z; z += kQuad) {
      const int b = block(z, lane0);
      if (kQuad == 4 && B % 4 == 0) {
        if (b < B) *reinterpret_cast<f32x4*>(row + b) = f32x4{x[z], x[z + 1 < Z ? z + 1 : 0], x[z + 2 < Z ? z + 2 : 0], x[z + 3 < Z ? z + 3 : 0]};
      } else {
#pragma unroll
        for (int i = 0; i < kQuad; ++i)
          if (b + i < B) row[b + i] = x[z + i];
      }
    }
  }
};

// x, a row's scores (-inf behind its end), becomes the probabilities; returns whether any score is above -inf.  NaN stays NaN.
template <int Z, int W>
__device__ __forceinline__ bool row_softmax(float* lds, float (&x)[Z], float& lse) {
  float top = x[0];
  bool any = false;
#pragma unroll
  for (int z = 0; z < Z; ++z) {
    any |= x[z] != -__builtin_inff();
    top = fmaxf(top, x[z]);
  }
  top = row_join<W>(wave_top(top), lds, [](float a, float b) { return fmaxf(a, b); });
  const float live = row_join<W>(__ballot(any) ? 1.f : 0.f, lds, [](float a, float b) { return a + b; });
  if (live == 0.f) return false;
  float sum = 0.f;
#pragma unroll
  for (int z = 0; z < Z; ++z) {
    // exp and log through powers of two, as the hardware has them: their arguments' rounding is off by 2^-24 of the distance to
    // the row's largest score, which is little where the probability is not
    x[z] = __builtin_amdgcn_exp2f((x[z] - top) * 1.44269504f);
    sum += x[z];
  }
  sum = row_join<W>(wave_total(sum), lds, [](float a, float b) { return a + b; });
  lse = top + __builtin_amdgcn_logf(sum) * 0.693147181f;
  const float inv = __builtin_amdgcn_rcpf(sum);
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

struct BalanceOut {
  int32_t *counts, *n_valid;
  float *prob, *loss;
  float balance, z;
};

// n tokens, sum of the squared log sums, sum over the blocks of counts times probabilities
__device__ __forceinline__ void balance_finish(const BalanceOut& out, int n, float lse2, float dot, int B, int e) {
  const float inv = n > 0 ? 1.f / (float)n : 0.f;
  const float lb = (float)B / (float)e * dot * inv * inv, lz = lse2 * inv;
  *out.n_valid = n;
  // a term of weight 0 is left out, so that an overflow of the other's does not reach the sum
  out.loss[0] = (out.balance != 0.f ? out.balance * lb : 0.f) + (out.z != 0.f ? out.z * lz : 0.f);
  out.loss[1] = lb;
  out.loss[2] = lz;
}

// Waves of a workgroup where a wave has a row to itself (W == 1): their probabilities meet in LDS.
constexpr int balance_rows(int w, int z) { return w > 1 ? 1 : z <= 4 ? 16 : 8; }
template <int Z, int W>
constexpr int balance_threads() { return 64 * W * balance_rows(W, Z); }

// A row is asked for while the one before is computed.  A workgroup that is alone (W == 1 only) finishes the loss itself.  LDS: counts [B] ints, then for W == 1 the waves' probabilities [waves][B].
template <int Z, int W>
__global__ __launch_bounds__((balance_threads<Z, W>())) void balance_part_kernel(const float* __restrict__ scores,
                                                                                 const int32_t* __restrict__ block_idx,
                                                                                 const uint8_t* __restrict__ valid, int n_tok, int B,
                                                                                 int e, BalancePart part, BalanceOut out) {
  typedef RowMap<Z, W> Map;
  extern __shared__ int32_t s_cnt[];
  constexpr int kThreads = balance_threads<Z, W>(), kRows = balance_rows(W, Z);
  __shared__ float s_join[16], s_lse2[16];
  __shared__ int32_t s_tok[16];
  const int tid = threadIdx.x, lane0 = W == 1 ? (tid & 63) : tid, slot = W == 1 ? tid / 64 : 0;
  for (int b = tid; b < B; b += kThreads) s_cnt[b] = 0;
  const bool alone = W == 1 && gridDim.x == 1;
  if (blockIdx.x == 0 && tid == 0 && !alone) *part.ticket = 0u;   // of the next launch
  __syncthreads();
  float acc[Z], next[Z], lse2 = 0.f;
  int n = 0, valid_next = 0, idx_next = -1;
#pragma unroll
  for (int z = 0; z < Z; ++z) acc[z] = next[z] = 0.f;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  auto load = [&](int64_t t) {
    if (t >= n_tok) return;
    valid_next = valid ? valid[t] : 1;
    if (lane0 < e) idx_next = block_idx[(size_t)t * e + lane0];
    Map::load(scores + (size_t)t * B, B, lane0, next);   // also of a row that pads the batch: it is not looked at
  };
  load((int64_t)blockIdx.x * kRows + slot);
  for (int64_t t = (int64_t)blockIdx.x * kRows + slot; t < n_tok; t += stride) {
    float x[Z], lse;
#pragma unroll
    for (int z = 0; z < Z; ++z) x[z] = next[z];
    const int on = valid_next, idx = idx_next;
    load(t + stride);
    if (!on || !row_softmax<Z, W>(s_join, x, lse)) continue;
#pragma unroll
    for (int z = 0; z < Z; ++z) acc[z] += x[z];
    lse2 += lse * lse;
    ++n;
    if (lane0 < e && (unsigned)idx < (unsigned)B) atomicAdd(&s_cnt[idx], 1);
    for (int q = lane0 + 64 * W; q < e; q += 64 * W) {
      const int b = block_idx[(size_t)t * e + q];
      if ((unsigned)b < (unsigned)B) atomicAdd(&s_cnt[b], 1);
    }
  }
  float* s_prob = reinterpret_cast<float*>(s_cnt + B);
  if constexpr (W == 1) {
#pragma unroll
    for (int z = 0; z < Z; ++z)
      if (Map::block(z, lane0) < B) s_prob[slot * B + Map::block(z, lane0)] = acc[z];
    if (lane0 == 0) { s_lse2[slot] = lse2; s_tok[slot] = n; }
  }
  __syncthreads();
  float* prob = alone ? out.prob : part.prob + (size_t)blockIdx.x * B;
  int32_t* count = alone ? out.counts : part.count + (size_t)blockIdx.x * B;
  if constexpr (W == 1) {
    float dot = 0.f;
    for (int b = tid; b < B; b += kThreads) {
      float p = 0.f;
#pragma unroll
      for (int w = 0; w < kRows; ++w) p += s_prob[w * B + b];
      prob[b] = p;
      dot += p * (float)s_cnt[b];
    }
    if (alone) {
      dot = wave_total(dot);
      if (lane0 == 0) s_join[slot] = dot;
      __syncthreads();
    }
    if (tid == 0) {
      lse2 = 0.f;
      n = 0;
#pragma unroll
      for (int w = 0; w < kRows; ++w) { lse2 += s_lse2[w]; n += s_tok[w]; }
      if (alone) {
        dot = 0.f;
#pragma unroll
        for (int w = 0; w < kRows; ++w) dot += s_join[w];
        balance_finish(out, n, lse2, dot, B, e);
      }
    }
  } else {
#pragma unroll
    for (int z = 0; z < Z; ++z)
      if (Map::block(z, lane0) < B) prob[Map::block(z, lane0)] = acc[z];
  }
  for (int b = tid; b < B; b += kThreads) count[b] = s_cnt[b];
  if (tid == 0 && !alone) { part.lse2[blockIdx.x] = lse2; part.tokens[blockIdx.x] = n; }
}

// Joins the workgroups' partial sums, 64 blocks and 16 groups of workgroups per workgroup of 1024 threads; the workgroup
// that is done last adds the others' shares of the loss up in order.
__global__ __launch_bounds__(1024) void balance_join_kernel(BalancePart part, int n_part, int B, int e, BalanceOut out) {
  __shared__ float s_prob[16][64], s_lse2[16];
  __shared__ int32_t s_cnt[16][64], s_tok[16];
  const int tid = threadIdx.x, lane = tid & 63, g = tid >> 6, b = blockIdx.x * 64 + lane;
  float p = 0.f, l2 = 0.f;
  int32_t c = 0, n = 0;
  if (b < B && g < n_part) {
    const size_t at = (size_t)g * B + b;
    p = sum_places(part.prob + at, (n_part - g + 15) / 16, (size_t)16 * B);
    c = sum_places(part.count + at, (n_part - g + 15) / 16, (size_t)16 * B);
  }
  if (tid < n_part) {   // at most 256 workgroups
    l2 = part.lse2[tid];
    n = part.tokens[tid];
  }
  s_prob[g][lane] = p;
  s_cnt[g][lane] = c;
  l2 = wave_sum(l2);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, kWave);
  if (lane == 0) { s_lse2[g] = l2; s_tok[g] = n; }
  __syncthreads();
  if (g != 0) return;
  p = 0.f;
  c = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) { p += s_prob[i][lane]; c += s_cnt[i][lane]; }
  if (b < B) { out.prob[b] = p; out.counts[b] = c; }
  float dot = wave_sum(p * (float)c);
  if (gridDim.x > 1) {
    uint32_t last = 0u;
    if (lane == 0) {
      __hip_atomic_store(&part.dot[blockIdx.x], dot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = __hip_atomic_fetch_add(part.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
    if (!__builtin_amdgcn_readfirstlane(last)) return;
    dot = 0.f;
    for (unsigned i = lane; i < gridDim.x; i += 64) dot += __hip_atomic_load(&part.dot[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    dot = wave_sum(dot);
  }
  if (lane == 0) {
    l2 = 0.f;
    n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) { l2 += s_lse2[i]; n += s_tok[i]; }
    balance_finish(out, n, l2, dot, B, e);
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
  typedef RowMap<Z, W> Map;
  __shared__ float s_join[16];
  constexpr int kRows = W == 1 ? 4 : 1;
  const int tid = threadIdx.x, lane0 = W == 1 ? (tid & 63) : tid, slot = W == 1 ? tid / 64 : 0;
  const int64_t first = (int64_t)blockIdx.x * kRows + slot, stride = (int64_t)gridDim.x * kRows;
  float next[Z], f[Z];
  int valid_next = 0;
#pragma unroll
  for (int z = 0; z < Z; ++z) next[z] = 0.f;
  auto load = [&](int64_t t) {
    if (t >= n_tok) return;
    valid_next = valid ? valid[t] : 1;
    Map::load(scores + (size_t)t * B, B, lane0, next);
  };
  load(first);
  const int n = *n_valid;
  const float inv = n > 0 ? 1.f / (float)n : 0.f, g = dloss ? *dloss : 1.f;
  const float cb = g * balance * (float)B * inv, cz = g * z_weight * 2.f * inv;
#pragma unroll
  for (int z = 0; z < Z; ++z) {
    const int b = Map::block(z, lane0);
    f[z] = b < B ? (float)counts[b] * (inv / (float)e) : 0.f;
  }
  for (int64_t t = first; t < n_tok; t += stride) {
    float x[Z], lse, mean = 0.f;
#pragma unroll
    for (int z = 0; z < Z; ++z) x[z] = next[z];
    const int on = valid_next;
    load(t + stride);
    const bool live = on && row_softmax<Z, W>(s_join, x, lse);
    if (live) {
#pragma unroll
      for (int z = 0; z < Z; ++z) mean += f[z] * x[z];
      mean = row_join<W>(wave_total(mean), s_join, [](float a, float b) { return a + b; });
    }
    const float lz = cz != 0.f && live ? cz * lse : 0.f;
#pragma unroll
    for (int z = 0; z < Z; ++z) x[z] = live ? x[z] * (cb * (f[z] - mean) + lz) : 0.f;
    Map::store(dscores + (size_t)t * B, B, lane0, x);
  }
}

}  // namespace meft
