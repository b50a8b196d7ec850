// Dropout whose mask is a function of the element's place: y = res + keep(t, c) * out * scale, forward and backward alike.
//
// The mask is that of Philox4x32 with 10 rounds (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011): the
// counter of columns 8 g .. 8 g + 7 of token t is (g, t, low word, high word of the offset), the key the seed.  Each of the
// four result words serves two columns with 16 bits each, the low ones first: an element is kept where its 16 bits are at
// least thr.  16 bits make the dropped share a multiple of 2^-16 (scale = 65536 / (65536 - thr) is the exact inverse of the
// kept one, so the expectation is that of `out`) and cost half the generator's multiplications of 32.
#pragma once
#include "common.h"
#include "tile_div.h"

namespace meft {

struct DropArgs {
  uint32_t k0, k1;               // seed
  uint64_t offset;
  const uint64_t* step;          // added to the offset where given: a captured launch draws anew in every replay
  uint32_t thr;                  // dropped where the 16 bits are below; 0: nothing is dropped
  float scale;
};

__device__ __forceinline__ uint64_t drop_offset(const DropArgs& a) { return a.offset + (a.step ? *a.step : 0ull); }

__device__ __forceinline__ u32x4 philox4x32(u32x4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
    c = u32x4{(uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a};
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

// v[j] = kept ? v[j] * scale : 0 for the eight columns of group g of token t
__device__ __forceinline__ void drop8(const DropArgs& a, uint64_t offset, uint32_t t, uint32_t g, float (&v)[8]) {
  const u32x4 w = philox4x32(u32x4{g, t, (uint32_t)offset, (uint32_t)(offset >> 32)}, a.k0, a.k1);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = (w[i] & 0xFFFFu) >= a.thr ? v[2 * i] * a.scale : 0.f;
    v[2 * i + 1] = (w[i] >> 16) >= a.thr ? v[2 * i + 1] * a.scale : 0.f;
  }
}

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
  // what was widened from the words is not kept beyond here: it is widened from them again
  __device__ __forceinline__ void forget() {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) asm volatile("" : "+v"(w[i]));
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

// eight elements; bf16 past L2 where asked
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8], bool past) {
  if constexpr (sizeof(T) == 2) {
    if (past) {
      asm volatile("");   // here and below: else the compiler makes one of the two stores, the ordinary one
      Vec16<T>::store(p, v);
      asm volatile("");
      return;
    }
  }
  Vec8<T>::store(p, v);
}

constexpr int kDropSpan = 256;   // groups of eight columns of a workgroup and round, one a thread

// Memory bounds it: 20 integer multiplications per eight elements hide behind their 32 to 48 bytes.  8192 x 4096 bf16, p 0.05:
// 37 us with a residual (5.4 TB/s; 42 with the result kept in L2), 25.7 without (5.2 TB/s); four groups a thread in a grid that
// covers them all took 47 and 31, results kept in L2.
// A workgroup walks spans of consecutive groups, asking for the next while one is computed.  step_t, step_g: the workgroups'
// stride in whole rows and groups.  y may be out or res: a thread reads its elements before it writes them.
template <typename T, bool kDrop>
__global__ __launch_bounds__(256) void dropout_add_kernel(const T* out, const T* res, T* y, int n_tok, int groups, uint32_t inv,
                                                          uint32_t step_t, uint32_t step_g, bool past, DropArgs a) {
  const uint64_t total = (uint64_t)n_tok * groups, stride = (uint64_t)gridDim.x * kDropSpan;
  uint64_t first = (uint64_t)blockIdx.x * kDropSpan;
  uint32_t t0 = (uint32_t)(first / (uint32_t)groups), g0 = (uint32_t)(first % (uint32_t)groups);
  const uint64_t offset = kDrop ? drop_offset(a) : 0;
  Raw8<T> raw_out, raw_res;
  auto load = [&](uint64_t at) {
    const uint64_t i = at + threadIdx.x;
    if (i >= total) return;
    raw_out.load(out + i * 8);
    if (res) raw_res.load(res + i * 8);
  };
  raw_out.clear();
  raw_res.clear();
  load(first);
  for (; first < total; first += stride) {
    float v[8], r[8];
    raw_out.widen(v);
    raw_res.widen(r);
    load(first + stride);
    const uint64_t i = first + threadIdx.x;
    if (kDrop) {
      const uint32_t w = g0 + threadIdx.x, dt = (uint32_t)tile_div((int)w, groups, inv);
      drop8(a, offset, t0 + dt, w - dt * groups, v);
    }
#pragma unroll
    for (int z = 0; z < 8; ++z) v[z] += r[z];
    if (i < total) store8(y + i * 8, v, past);
    t0 += step_t;
    g0 += step_g;
    if (g0 >= (uint32_t)groups) {
      g0 -= groups;
      ++t0;
    }
  }
}

}  // namespace meft
