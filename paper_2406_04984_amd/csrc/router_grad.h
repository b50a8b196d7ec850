// The router's gradient: from the gradient of its scores p[t, b] = Wg[b, :] . h[t, :] + bias[b]
//
//   dh[t, :] = add[t, :] + sum_b ds[t, b] Wg[b, :]      dWg[b, :] = sum_t ds[t, b] h[t, :]      dbias[b] = sum_t ds[t, b]
//
// Both contractions are far below the matrix cores' rate at the number of blocks in use (4 T d B flop against 6 T d bytes at
// bf16): reading h and add and writing dh bounds them.  The wide operands (h, the router) are loaded as four consecutive columns
// of eight rows per lane straight into registers, where swapping halves of words gives the matrix instruction's operand
// (it wants eight rows of one column per lane); lane l then holds columns 4 (l % 32) + j of its four result tiles j, so that a
// result row leaves as one 8- or 16-byte word per lane, 32 lanes on consecutive addresses.
//
// 8192 x 4096 bf16, 64 blocks: 49 us for 217 MB (4.4 TB/s; a copy in tiles of this shape reaches 5.0 to 5.3) and 5.0 for the join;
// 4096 x 4096, 256 blocks: 67 and 8 us, there bound by the instructions of dWg's waves and by their loads through the vector cache.
//
// ds arrives in fp32.  bf16 shapes cut it in three bf16 parts of eight bits each, which together are ds (below 2^-110 up to the last bits
// that bf16's range has), and multiply all three: the products are those of fp32.  Two parts took 47 and 53 us there and kept 16 bits.
// fp32 shapes use fp32 matrix instructions.
#pragma once
#include "common.h"

namespace meft {

// eight rows of four columns, and the operands that they give
template <typename T>
struct Rows8;

template <>
struct Rows8<bf16_t> {
  typedef u32x2 Quad;
  Quad w[8];
  static __device__ __forceinline__ Quad load(__amdgpu_buffer_rsrc_t r, uint32_t at) {
    return __builtin_bit_cast(Quad, __builtin_amdgcn_raw_buffer_load_b64(r, (int)at, 0, 0));
  }
  static __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t r, uint32_t at, const float (&v)[4]) {
    const Quad q = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    __builtin_amdgcn_raw_buffer_store_b64(q, r, (int)at, 0, 0);
  }
  // the eight rows of column j
  __device__ __forceinline__ bf16x8 operand(int j) const {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r[i] = __builtin_amdgcn_perm(w[2 * i + 1][j / 2], w[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
    return __builtin_bit_cast(bf16x8, r);
  }
  static __device__ __forceinline__ void widen(Quad q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xFFFF0000u);
    v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xFFFF0000u);
  }
};

template <>
struct Rows8<float> {
  typedef f32x4 Quad;
  Quad w[8];
  static __device__ __forceinline__ Quad load(__amdgpu_buffer_rsrc_t r, uint32_t at) {
    return __builtin_bit_cast(Quad, __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, 0));
  }
  static __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t r, uint32_t at, const float (&v)[4]) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]}), r, (int)at, 0, 0);
  }
  static __device__ __forceinline__ void widen(Quad q, float (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = q[j];
  }
};

// The three bf16 parts of eight values: the upper half of a value's word, of what is left of it, and of what is left then.  They are cut
// and not rounded: each difference is exact, and the largest values do not round to an infinity.
__device__ __forceinline__ void split(const float (&a)[8], bf16x8 (&part)[3]) {
  u32x4 w[3];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[2] = {a[2 * i], a[2 * i + 1]};
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      w[k][i] = __builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u);
#pragma unroll
      for (int j = 0; j < 2; ++j) x[j] -= __uint_as_float(__float_as_uint(x[j]) & 0xFFFF0000u);
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) part[k] = __builtin_bit_cast(bf16x8, w[k]);
}

// acc[j] += a (8 values of a row of the left operand per lane) * rows, for the four columns j
__device__ __forceinline__ void mma_rows8(const float (&a)[8], const Rows8<bf16_t>& rows, f32x16 (&acc)[4]) {
  bf16x8 part[3];
  split(a, part);
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(part[k], rows.operand(j), acc[j], 0, 0, 0);
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
constexpr int kRgWaves = 4;

template <typename T>
struct RouteGradArgs {
  const T *h, *Wg, *add;
  const float* ds;
  T *dh, *dWg;
  float *dbias, *part, *part_bias;   // part: [split][B][d], where there is more than one split
  int n_tok, d, B;
  int m_shift, splits, per_split;    // dWg: 2^m_shift waves along the blocks, splits of the tokens, tokens of a split (a multiple of 16)
  int dh_words;                      // of 16 bytes, the router's part of LDS; ds is behind it
  int n_dw, dw_slices, n_along;      // workgroups of dWg, their slices of columns (1 where only dbias is wanted); dh's along the tokens
};

template <typename T>
__device__ __forceinline__ void store4(T* p, const float (&v)[4]) {
  if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
}
// `rows` rows of `row_bytes` bytes from `base` on, which is the same in all lanes: what lies behind reads as 0 and is not
// written.  The rows of a tile, so far below 4 GB.
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const T* base, int rows, uint32_t row_bytes) {
  // the compiler does not always see that they are, and would then loop over the lanes
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)p), hi = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32));
  const int bytes = __builtin_amdgcn_readfirstlane((int)(max(rows, 0) * row_bytes));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((uint64_t)hi << 32 | lo), 0, bytes, 0x00020000);
}
constexpr uint32_t kNoColumn = 0xF0000000u;   // an offset behind the rows of any tile, also with a row's offset added

// A step of 16 blocks of ds in LDS, 128 words of 16 bytes: put as four blocks 4 q .. 4 q + 3 (q < 4) of a token, got as the eight of
// its lane's row of the left operand.
__device__ __forceinline__ void put_ds(u32x4* step, int row, int q, u32x4 x) { step[(q & 1) * 64 + (q >> 1) * 32 + row] = x; }
__device__ __forceinline__ void get_ds(const u32x4* step, int lane, float (&x)[8]) {
  const u32x4 w[2] = {step[lane], step[64 + lane]};
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i / 4][i % 4]);
}

// A step of 16 blocks of the router in LDS, as the matrix instructions want it: kUnits words of 16 bytes per lane.
template <typename T>
struct StepWords;
template <>
struct StepWords<bf16_t> {
  static constexpr int kUnits = 4;   // one per column j: its eight rows
  static __device__ __forceinline__ void put(u32x4* lds, const Rows8<bf16_t>& w, int lane) {
#pragma unroll
    for (int j = 0; j < 4; ++j) lds[j * 64 + lane] = __builtin_bit_cast(u32x4, w.operand(j));
  }
  static __device__ __forceinline__ void mma(const u32x4* step, const u32x4* lds, int lane, f32x16 (&acc)[4]) {
    float x[8];
    get_ds(step, lane, x);
    bf16x8 part[3];
    split(x, part);
    bf16x8 b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = __builtin_bit_cast(bf16x8, lds[j * 64 + lane]);
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(part[k], b[j], acc[j], 0, 0, 0);
  }
};
template <>
struct StepWords<float> {
  static constexpr int kUnits = 8;   // one per row u: its four columns
  static __device__ __forceinline__ void put(u32x4* lds, const Rows8<float>& w, int lane) {
#pragma unroll
    for (int u = 0; u < 8; ++u) lds[u * 64 + lane] = __builtin_bit_cast(u32x4, w.w[u]);
  }
  static __device__ __forceinline__ void mma(const u32x4* step, const u32x4* lds, int lane, f32x16 (&acc)[4]) {
    float x[8];
    get_ds(step, lane, x);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const f32x4 b = __builtin_bit_cast(f32x4, lds[u * 64 + lane]);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[u], b[j], acc[j], 0, 0, 0);
    }
  }
};

// steps of ds in registers or on their way: as many as 64 blocks have, half where a step takes eight times as long
template <typename T>
constexpr int dh_ahead() { return sizeof(T) == 2 ? 4 : 2; }
// steps of 16 blocks, rounded up to whole groups of those: what is behind the last block is 0
template <typename T>
constexpr int dh_steps(int n_blocks) { return (n_blocks + 16 * dh_ahead<T>() - 1) / (16 * dh_ahead<T>()) * dh_ahead<T>(); }
constexpr int kDhLds = 128 << 10;   // most of LDS that a workgroup's part of the router takes
constexpr int kDhDsLds = kRgWaves * 2 * 128 * 16;   // two steps of ds for each wave
template <typename T>
constexpr int dh_step_bytes() { return StepWords<T>::kUnits * 64 * 16; }

// dh.  A workgroup holds the router's rows of 128 columns in LDS, as operands, and walks tiles of 32 tokens per wave.  What is
// added to a tile and its ds are asked for while the tile before is computed.  More blocks than kDhLds holds are staged piece by
// piece for every tile.  `along` of `n_along` workgroups along the tokens.  kQuads: the number of blocks is a multiple of 4.
// kPieces: they are more than one group of steps.
template <typename T, bool kQuads, bool kPieces>
__device__ __forceinline__ void route_dh(const RouteGradArgs<T>& a, int along, int n_along, int slice, u32x4* s_w) {
  typedef Rows8<T> Rows;
  typedef StepWords<T> Words;
  constexpr int kMaxSteps = kDhLds / dh_step_bytes<T>();
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = slice * kRgCols + 4 * col;
  const uint32_t row_bytes = a.d * (uint32_t)sizeof(T), c_bytes = (uint32_t)min(c, a.d - 4) * (uint32_t)sizeof(T);
  constexpr int kAhead = dh_ahead<T>();
  const int steps = dh_steps<T>(a.B);
  const uint32_t o = 4 * half * row_bytes + (c < a.d ? c_bytes : kNoColumn);

  auto stage = [&](int first, int n) {   // steps first .. first + n - 1 of the router
    for (int s = wave; s < n; s += kRgWaves) {
      const int b0 = (first + s) * 16;
      const __amdgpu_buffer_rsrc_t wg = rows_at(a.Wg + (size_t)b0 * a.d, min(a.B - b0, 16), row_bytes);
      Rows w;
#pragma unroll
      for (int u = 0; u < 8; ++u) w.w[u] = Rows::load(wg, 8 * half * row_bytes + c_bytes + u * row_bytes);
      Words::put(s_w + s * Words::kUnits * 64, w, lane);
    }
  };
  // Two steps of ds, 32 blocks of 32 tokens: eight lanes a row, so that a load takes whole lines (a row per lane, as the operand
  // has them, touches as many lines as a load has lanes times a quarter).  Blocks and tokens that are not there are 0.
  auto load_ds = [&](__amdgpu_buffer_rsrc_t ds, int s, u32x4(&x)[4]) {
    const int b = 16 * s + 4 * (lane & 7);
    const uint32_t at = (uint32_t)(lane >> 3) * a.B * 4u + b * 4u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t o8 = at + 8u * i * a.B * 4u;
      if (kQuads) {
        x[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(ds, (int)(b < a.B ? o8 : kNoColumn), 0, 0));
      } else {   // a word of four might run over the row's end
#pragma unroll
        for (int u = 0; u < 4; ++u) x[i][u] = __builtin_amdgcn_raw_buffer_load_b32(ds, (int)(b + u < a.B ? o8 + 4 * u : kNoColumn), 0, 0);
      }
    }
  };
  const int64_t tile0 = (int64_t)along * kRgWaves + wave, n_tiles = ((int64_t)a.n_tok + 31) / 32;
  const int stride = n_along * kRgWaves;
  auto tile_rows = [&](int64_t tile) { return tile < 0 ? 0 : (int)max((int64_t)0, min((int64_t)32, a.n_tok - tile * 32)); };
  auto ds_of = [&](int64_t tile) { return rows_at(a.ds + (size_t)tile * 32 * a.B, tile_rows(tile), a.B * 4u); };

  u32x4 x[kAhead / 2][4];
  u32x4* const s_ds = s_w + a.dh_words + wave * (2 * 128);   // this wave's
  typename Rows::Quad y[16];   // 0 where nothing is added
  auto load_add = [&](int64_t tile) {
    const __amdgpu_buffer_rsrc_t add = rows_at(a.add + (a.add ? (size_t)tile * 32 * a.d : 0), a.add ? tile_rows(tile) : 0, row_bytes);
#pragma unroll
    for (int r = 0; r < 16; ++r) y[r] = Rows::load(add, o + (uint32_t)tile_row(r, 0) * row_bytes);
  };
  f32x16 acc[4];
  // kAhead steps from s0 on, whose router is at `w`; their places in x then take the same steps of another part or tile
  auto group = [&](const u32x4* w, __amdgpu_buffer_rsrc_t next, int next_s0, bool real = true) {
#pragma unroll
    for (int i = 0; i < kAhead / 2; ++i) {
      wave_lds_fence();
#pragma unroll
      for (int k = 0; k < 4; ++k) put_ds(s_ds + (lane >> 2 & 1) * 128, 8 * k + (lane >> 3), lane & 3, x[i][k]);
      load_ds(next, next_s0 + 2 * i, x[i]);
      wave_lds_fence();
      if (real) {
#pragma unroll
        for (int k = 0; k < 2; ++k) Words::mma(s_ds + k * 128, w + (2 * i + k) * Words::kUnits * 64, lane, acc);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto clear = [&] {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;
  };
  auto finish = [&](int64_t tile) {
    const __amdgpu_buffer_rsrc_t to = rows_at(a.dh + (size_t)tile * 32 * a.d, tile_rows(tile), row_bytes);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float v[4];
      Rows::widen(y[r], v);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += acc[j][r];
      Rows::store(to, o + (uint32_t)tile_row(r, 0) * row_bytes, v);
    }
    __builtin_amdgcn_sched_barrier(0);
    load_add(tile + stride);
    __builtin_amdgcn_sched_barrier(0);
  };
  if constexpr (kPieces) {
    const int pieces = (steps + kMaxSteps - 1) / kMaxSteps;
    if (pieces == 1) stage(0, steps);
#pragma unroll
    for (int i = 0; i < kAhead / 2; ++i) load_ds(ds_of(tile0), 2 * i, x[i]);
    load_add(tile0);
    if (pieces == 1) __syncthreads();
    // every wave of the workgroup makes as many rounds as the first: there may be barriers in them
    for (int64_t tile = tile0; tile - wave < n_tiles; tile += stride) {
      const __amdgpu_buffer_rsrc_t ds = ds_of(tile), ds_next = ds_of(tile + stride);
      clear();
      for (int p = 0; p < pieces; ++p) {
        const int first = p * kMaxSteps, n = min(steps - first, kMaxSteps);
        if (pieces > 1) {
          __syncthreads();
          stage(first, n);
          __syncthreads();
        }
        for (int s0 = 0; s0 < n; s0 += kAhead) {
          const bool same = first + s0 + kAhead < steps;
          group(s_w + s0 * Words::kUnits * 64, same ? ds : ds_next, same ? first + s0 + kAhead : 0);
        }
      }
      finish(tile);
    }
  } else {
    // One round more than there are tiles, the first of a tile before the first one: nothing of it is there, and the loop's
    // waits for operands are then those of its steady state.
    stage(0, kAhead);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAhead / 2; ++i) x[i][0] = x[i][1] = x[i][2] = x[i][3] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int r = 0; r < 16; ++r) y[r] = typename Rows::Quad{};
    for (int64_t tile = tile0 - stride; tile < n_tiles; tile += stride) {
      clear();
      group(s_w, ds_of(tile + stride), 0, tile >= tile0);
      finish(tile);
    }
  }
}

// dWg and dbias.  A wave: 32 M blocks x 128 columns over a share of the tokens, 16 at a time, the next step's operands on their
// way; 2^m_shift waves lie along the blocks, the others share out the tokens and are added through LDS.
template <typename T, int M, bool kBias>
__device__ __forceinline__ void route_dw(const RouteGradArgs<T>& a, int split, int slice, int group, float* lds) {
  typedef Rows8<T> Rows;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m_waves = 1 << a.m_shift, k_waves = kRgWaves >> a.m_shift, mw = wave & (m_waves - 1), kw = wave >> a.m_shift;
  const int b0 = (group * m_waves + mw) * 32 * M;
  const int c = slice * kRgCols + 4 * (lane & 31);
  const int64_t begin = (int64_t)split * a.per_split;
  const int len = (int)min((int64_t)a.per_split, a.n_tok - begin);   // tokens of this split
  const uint32_t row_bytes = a.d * (uint32_t)sizeof(T), ds_bytes = a.B * 4u;
  const uint32_t h_off = 8 * half * row_bytes + (uint32_t)min(c, a.d - 4) * (uint32_t)sizeof(T);
  uint32_t ds_off[M];
  f32x16 acc[M][4];
  float bias[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    ds_off[m] = 8 * half * ds_bytes + (uint32_t)min(b0 + 32 * m + (lane & 31), a.B - 1) * 4u;
    bias[m] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[m][j][r] = 0.f;
  }
  constexpr int kAhead = 2;   // steps whose operands are in registers or on their way
  Rows rows[kAhead];
  float x[kAhead][M][8];
  const int stride = 16 * k_waves;
  auto load = [&](int t0, Rows& w, float(&v)[M][8]) {   // tokens that are not there are 0
    const int left = min(len - t0, 16);
    const __amdgpu_buffer_rsrc_t h = rows_at(a.h + (size_t)(begin + t0) * a.d, left, row_bytes);
    const __amdgpu_buffer_rsrc_t ds = rows_at(a.ds + (size_t)(begin + t0) * a.B, left, ds_bytes);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      w.w[u] = Rows::load(h, h_off + u * row_bytes);
#pragma unroll
      for (int m = 0; m < M; ++m)
        v[m][u] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(ds, (int)(ds_off[m] + u * ds_bytes), 0, 0));
    }
  };
  auto step = [&](const Rows& w, const float(&v)[M][8]) {
#pragma unroll
    for (int m = 0; m < M; ++m) {
      mma_rows8(v[m], w, acc[m]);
      if (kBias) bias[m] += ((v[m][0] + v[m][1]) + (v[m][2] + v[m][3])) + ((v[m][4] + v[m][5]) + (v[m][6] + v[m][7]));
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead - 1; ++i) load(16 * kw + i * stride, rows[i], x[i]);
  for (int t0 = 16 * kw; t0 < len; t0 += kAhead * stride) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      load(t0 + (i + kAhead - 1) * stride, rows[(i + kAhead - 1) % kAhead], x[(i + kAhead - 1) % kAhead]);
      __builtin_amdgcn_sched_barrier(0);   // the compiler would ask for a step's operands at the end of the step before
      step(rows[i], x[i]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // the waves that shared out the tokens, in pairs
  for (int n = k_waves / 2; n > 0; n /= 2) {
    __syncthreads();
    float* s = lds + ((kw & (n - 1)) * m_waves + mw) * (M * 64 * 64) + lane;
    if (kw >= n && kw < 2 * n) {
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[((m * 4 + j) * 16 + r) * 64] = acc[m][j][r];
    }
    __syncthreads();
    if (kw < n) {
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[m][j][r] += s[((m * 4 + j) * 16 + r) * 64];
    }
  }
  if (kBias) {
    __syncthreads();
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const float v = bias[m] + __shfl_xor(bias[m], 32, kWave);
      if (half == 0) lds[(wave * M + m) * 32 + lane] = v;
    }
    __syncthreads();
    if (kw == 0 && half == 0) {
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const int b = b0 + 32 * m + lane;
        float v = 0.f;
        for (int k = 0; k < k_waves; ++k) v += lds[((k * m_waves + mw) * M + m) * 32 + lane];
        if (b < a.B) (a.splits > 1 ? a.part_bias + (size_t)split * a.B : a.dbias)[b] = v;
      }
    }
  }
  if (kw != 0 || !a.dWg) return;
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const int first = b0 + 32 * m, left = min(a.B - first, 32);
    if (a.splits > 1) {
      const __amdgpu_buffer_rsrc_t to = rows_at(a.part + ((size_t)split * a.B + first) * a.d, left, a.d * 4u);
      const uint32_t o = 4 * half * a.d * 4u + (c < a.d ? c * 4u : kNoColumn);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        Rows8<float>::store(to, o + (uint32_t)tile_row(r, 0) * a.d * 4u, {acc[m][0][r], acc[m][1][r], acc[m][2][r], acc[m][3][r]});
    } else {
      const __amdgpu_buffer_rsrc_t to = rows_at(a.dWg + (size_t)first * a.d, left, row_bytes);
      const uint32_t o = 4 * half * row_bytes + (c < a.d ? c * (uint32_t)sizeof(T) : kNoColumn);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        Rows::store(to, o + (uint32_t)tile_row(r, 0) * row_bytes, {acc[m][0][r], acc[m][1][r], acc[m][2][r], acc[m][3][r]});
    }
  }
}

// Both in one launch, so that neither's start and end leave the memory idle: the first n_dw workgroups compute dWg, the others dh.
// Along the tokens fastest, so that the slices of the same tokens share an XCD's L2.
template <typename T, int M>
__global__ __launch_bounds__(64 * kRgWaves, 2) void route_grad_kernel(RouteGradArgs<T> a) {
  extern __shared__ u32x4 s_lds[];
  const int id = blockIdx.x;
  if (id < a.n_dw) {
    const int rest = __builtin_amdgcn_readfirstlane(id / a.splits), group = __builtin_amdgcn_readfirstlane(rest / a.dw_slices);
    const int split = id - rest * a.splits, slice = rest - group * a.dw_slices;
    if (slice == 0 && a.dbias) route_dw<T, M, true>(a, split, slice, group, reinterpret_cast<float*>(s_lds));
    else route_dw<T, M, false>(a, split, slice, group, reinterpret_cast<float*>(s_lds));
  } else {
    const int i = id - a.n_dw, slice = __builtin_amdgcn_readfirstlane(i / a.n_along), along = i - slice * a.n_along;
    if (dh_steps<T>(a.B) == dh_ahead<T>()) {
      if (a.B % 4 == 0) route_dh<T, true, false>(a, along, a.n_along, slice, s_lds);
      else route_dh<T, false, false>(a, along, a.n_along, slice, s_lds);
    } else {
      if (a.B % 4 == 0) route_dh<T, true, true>(a, along, a.n_along, slice, s_lds);
      else route_dh<T, false, true>(a, along, a.n_along, slice, s_lds);
    }
  }
}

// the splits of dWg and dbias added up, in order; one workgroup more than dWg's quadruples need writes dbias
template <typename T>
__global__ __launch_bounds__(256) void route_dw_join_kernel(RouteGradArgs<T> a) {
  const int64_t n = (int64_t)a.B * a.d, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (a.dbias && blockIdx.x == gridDim.x - 1)
    for (int b = threadIdx.x; b < a.B; b += 256) a.dbias[b] = sum_places(a.part_bias + b, a.splits, a.B);
  if (i >= n || !a.dWg) return;
  const f32x4 v = sum_places(reinterpret_cast<const f32x4*>(a.part + i), a.splits, (size_t)(n / 4));
  store4(a.dWg + i, {v[0], v[1], v[2], v[3]});
}

}  // namespace meft
