// Host side of the calls around the layer (include/meft.h): norms, dropout, the router's balance loss and its gradient.
// Argument validation, workspace layout and launches; the kernels are in the headers included below.
#include <cmath>
#include <initializer_list>
#include <mutex>

#include "balance.h"
#include "dropout.h"
#include "host.h"
#include "norm.h"
#include "router_grad.h"

namespace meft {
namespace {

constexpr int kCus = 256;   // compute units of an MI355X

template <typename T>
bool aligned_as(const void* p) { return reinterpret_cast<uintptr_t>(p) % alignof(T) == 0; }
bool ok16(const void* p) { return p && aligned16(p); }
bool null_or16(const void* p) { return !p || aligned16(p); }

// An operand's bytes.  Outputs share none with each other or with an input that is read while they are written; one that the
// header lets stand in an input's place starts where it does.
struct Span {
  const void* p;
  size_t bytes;
  bool shares(const Span& o) const {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(o.p);
    return p && o.p && bytes && o.bytes && (a < b ? b - a < bytes : a - b < o.bytes);
  }
};
// the first `in_place` of the outputs may stand in the place of one of `places`
bool outputs_apart(std::initializer_list<Span> outs, int in_place, std::initializer_list<Span> ins, std::initializer_list<Span> places) {
  int i = 0;
  for (const Span* o = outs.begin(); o != outs.end(); ++o, ++i) {
    for (const Span* other = outs.begin(); other != o; ++other)
      if (o->shares(*other)) return false;
    for (const Span& in : ins)
      if (o->shares(in)) return false;
    for (const Span& in : places)
      if (o->shares(in) && (i >= in_place || o->p != in.p)) return false;
  }
  return true;
}
size_t row_bytes(const meft_shape& s) { return (size_t)s.d * (s.dtype == MEFT_BF16 ? 2 : 4); }

// ---- norms ----------------------------------------------------------------------------------
// Groups of eight columns per lane and waves per row: two groups where they spare waves, and with them barriers, as far as the
// backward's registers allow it.  Forward + backward, us: d 768, 16384 tokens bf16, two groups in one wave / one in two 28.4 / 30.3;
// d 8192, 4096 tokens, two in eight / one in sixteen 72.4 / 78.4.  At d 4096 one group in eight waves lets a compute unit hold
// twice the rows (64 tokens, backward: 3.3 us against 4.2 of two in four; 8192 tokens with dropout 57 / 59).
struct NormShape {
  int v, w;
};
NormShape norm_shape(int d) {
  const int groups = d / 8;
  if (groups <= 64) return {1, 1};
  if (groups <= 128) return {2, 1};
  if (groups <= 256) return {1, 4};
  if (groups <= 512) return {1, 8};
  if (groups <= 1024) return {2, 8};
  return {2, 16};
}

// Rows of a workgroup: as many as leave every compute unit a workgroup.
int norm_slots(const meft_shape& s) {
  int slots = norm_max_slots(norm_shape(s.d).w);
  while (slots > 1 && ((int64_t)s.T + slots - 1) / slots < kCus) slots /= 2;
  return slots;
}
int norm_grid(const meft_shape& s, int most) {
  const int slots = norm_slots(s);
  const int64_t need = ((int64_t)s.T + slots - 1) / slots;
  return (int)(need < 1 ? 1 : need < most ? need : most);
}
// Workgroups of the backward, each of which leaves partial sums of dgamma and dbeta: at least eight rows for each slot before a
// compute unit gets a second workgroup (layer kind with dropout, d 4096, us, 256 / 512 of them: 2003 tokens 18.7 / 20.2, 8192
// tokens 63 / 60).
int norm_bwd_grid(const meft_shape& s) {
  const int64_t eight = (int64_t)s.T / (8 * norm_slots(s));
  return norm_grid(s, eight < kCus ? kCus : eight < 2 * kCus ? (int)eight : 2 * kCus);
}
// Few rows: the weights' gradients apart, in one launch with dx.  Forward + backward, us, apart / two launches: 128 x 768 fp32 13.1 /
// 16.3, 512 x 768 fp32 12.3 / 15.3, 512 x 4096 bf16 14.4 / 16.1; wider rows 16 x 8192 bf16 12.7 / 16.4, 512 x 8192 bf16 18.4 / 20.5,
// 512 x 8192 fp32 29.5 / 30.3, 512 x 16384 fp32 61.5 / 98.3; more rows 1000 x 4096 22.0 / 19.3, and 1000 x 768 fp32 14.9 / 15.9 with
// 10.9 us on the device instead of 8.9.
bool norm_columns_apart(const meft_shape& s) { return s.T > 0 && s.T <= 512; }
int norm_apart_rows(const meft_shape& s) {
  const int slots = norm_max_slots(norm_shape(s.d).w);
  return (int)(((int64_t)s.T + slots - 1) / slots);
}

// The forward: 16 waves for every compute unit, each with a few rows to ask for ahead (workgroups per compute unit, us: eight-wave
// ones, 2003 x 4096 with dropout, 2 / 8: 15.1 / 16.1, 4096 x 4096 fp32 24.2 / 27; four-wave ones, 8192 x 2048, 2 / 4: 17.1 / 13.8).
int norm_fwd_grid(const meft_shape& s) { return norm_grid(s, norm_shape(s.d).w >= 8 ? 2 * kCus : 4 * kCus); }

#define MEFT_NORM_SHAPES(X) X(1, 1) X(2, 1) X(1, 4) X(1, 8) X(2, 8) X(2, 16)

template <typename T, int kMode>
void launch_norm_fwd(const meft_shape& s, const NormFwdArgs<T>& a, hipStream_t st) {
  const NormShape n = norm_shape(s.d);
  const dim3 grid(norm_fwd_grid(s)), block(64 * n.w * norm_slots(s));
#define X(V, W) \
  if (n.v == V && n.w == W) MEFT_LAUNCH("norm_fwd", (norm_fwd_kernel<T, V, W, kMode>), grid, block, 0, st, a);
  MEFT_NORM_SHAPES(X)
#undef X
}

template <typename T, int kMode, int kGrads>
void launch_norm_bwd(const meft_shape& s, const NormBwdArgs<T>& a, hipStream_t st) {
  const NormShape n = norm_shape(s.d);
  const dim3 grid(kGrads == 3 ? a.row_wgs + (s.d + kApartCols - 1) / kApartCols : norm_bwd_grid(s));
  const dim3 block(64 * n.w * (kGrads == 3 ? norm_max_slots(n.w) : norm_slots(s)));
#define X(V, W) \
  if (n.v == V && n.w == W) MEFT_LAUNCH("norm_bwd", (norm_bwd_kernel<T, V, W, kMode, kGrads>), grid, block, 0, st, a);
  MEFT_NORM_SHAPES(X)
#undef X
}

// Large results go past L2.  us, past / kept, one card, the mean of three runs each: dropout with the residual add 8192 x 4096 bf16
// 62.5 / 65.8; plain norm, forward + backward, bf16: rms 8192 x 4096 74.3 / 76.7, layer 8192 x 4096 75.6 / 79.6, layer 16384 x 1024
// 39.1 / 42.5, rms 4096 x 8192 77.7 / 81.5.  Kept in L2: fp32 (layer 4096 x 4096 81.1 / 78.9) and the two results of add and norm
// (8192 x 4096 bf16 115.5 / 115.1).
bool past_l2(const meft_shape& s) { return s.dtype == MEFT_BF16 && (int64_t)s.T * s.d * 2 >= (int64_t)32 << 20; }

bool norm_ok(const meft_norm* n) {
  return n && (n->kind == MEFT_NORM_LAYER || n->kind == MEFT_NORM_RMS) && n->eps >= 0.f && std::isfinite(n->eps);
}

// 0 where nothing is dropped; -1: not a valid share
int drop_threshold(const meft_drop* d) {
  if (!d) return 0;
  if (!(d->p >= 0.f && d->p < 1.f)) return -1;
  const int thr = (int)std::floor((double)d->p * 65536.0 + 0.5);
  return thr <= 65535 ? thr : -1;
}

DropArgs drop_args(const meft_drop* d, const uint64_t* step, int thr) {
  DropArgs a{};
  if (d) {
    a.k0 = (uint32_t)d->seed;
    a.k1 = (uint32_t)(d->seed >> 32);
    a.offset = d->offset;
  }
  a.step = step;
  a.thr = (uint32_t)thr;
  a.scale = (float)(65536.0 / (65536.0 - thr));
  return a;
}

template <typename T>
meft_status norm_fwd(const meft_shape& s, const meft_norm& n, int mode, const DropArgs& drop, const void* x, const void* out,
                     const void* gamma, const void* beta, void* y, void* h, float* mean, float* rstd, hipStream_t st) {
  const NormFwdArgs<T> a{static_cast<const T*>(x), static_cast<const T*>(out), static_cast<const T*>(gamma), static_cast<const T*>(beta),
                         static_cast<T*>(y), static_cast<T*>(h), mean, rstd, s.T, s.d, n.kind == MEFT_NORM_LAYER,
                         (float)(1.0 / s.d), n.eps, past_l2(s), drop};
  if (mode == kNormPlain) launch_norm_fwd<T, kNormPlain>(s, a, st);
  else if (mode == kNormAdd) launch_norm_fwd<T, kNormAdd>(s, a, st);
  else launch_norm_fwd<T, kNormDrop>(s, a, st);
  return launch_status();
}

struct NormBwdWs {
  float* part;
  size_t bytes;
  NormBwdWs(const meft_shape& s, void* ws) {
    Carver c(ws);
    part = c.take<float>((size_t)norm_bwd_grid(s) * 2 * s.d);
    bytes = c.off;
  }
};

template <typename T, int kMode>
void norm_bwd_grads(const meft_shape& s, const NormBwdArgs<T>& a, int grads, hipStream_t st) {
  if (grads == 0) launch_norm_bwd<T, kMode, 0>(s, a, st);
  else if (grads == 1) launch_norm_bwd<T, kMode, 1>(s, a, st);
  else if (grads == 2) launch_norm_bwd<T, kMode, 2>(s, a, st);
  else launch_norm_bwd<T, kMode, 3>(s, a, st);
}

template <typename T>
meft_status norm_bwd(const meft_shape& s, const meft_norm& n, int mode, const DropArgs& drop, const void* y, const void* gamma,
                     const float* mean, const float* rstd, const void* dh, const void* dy, void* dx, void* dout, void* dgamma,
                     void* dbeta, void* ws, hipStream_t st) {
  const NormBwdWs w(s, ws);
  // the workgroups of the gradients read dh while dx is written: not where one stands in the other's place
  const bool apart = dgamma && norm_columns_apart(s) && dx != dh && dout != dh;
  const int grads = !dgamma ? 0 : apart ? 3 : dbeta ? 2 : 1;
  if (s.T == 0 && grads == 0) return MEFT_OK;
  const NormBwdArgs<T> a{static_cast<const T*>(y), static_cast<const T*>(gamma), static_cast<const T*>(dh), static_cast<const T*>(dy),
                         mean, rstd, static_cast<T*>(dx), static_cast<T*>(dout), w.part, static_cast<T*>(dgamma), static_cast<T*>(dbeta),
                         norm_apart_rows(s), s.T, s.d, n.kind == MEFT_NORM_LAYER,
                         (float)(1.0 / s.d), past_l2(s), drop};
  if (mode == kNormPlain) norm_bwd_grads<T, kNormPlain>(s, a, grads, st);
  else if (mode == kNormAdd) norm_bwd_grads<T, kNormAdd>(s, a, grads, st);
  else norm_bwd_grads<T, kNormDrop>(s, a, grads, st);
  if (grads == 1 || grads == 2)
    MEFT_LAUNCH("norm_grad", norm_grad_kernel<T>, dim3((s.d + 31) / 32, grads), dim3(512), 0, st, w.part, norm_bwd_grid(s), s.d,
                static_cast<T*>(dgamma), static_cast<T*>(dbeta));
  return launch_status();
}

constexpr int kDropWgs = 8 * kCus;   // workgroups of dropout_add at most

// ---- balance --------------------------------------------------------------------------------
// waves of a row of scores, and the scores of a lane
int balance_waves(const meft_shape& s) { return s.n_blocks <= 1024 ? 1 : 16; }
// Few rows for each wave of one workgroup: it is alone and finishes the loss, one launch less (forward + backward, us, alone / with
// the join: 128 tokens, 64 blocks 13.0 / 16.9, 256 blocks 13.3 / 16.1; 16 tokens, 1000 blocks 12.6 / 15.6, 64 tokens 18.1 / 16.8).
int balance_grid(const meft_shape& s) {
  const int rows = balance_rows(balance_waves(s), s.n_blocks <= 256 ? 4 : 16);
  if (balance_waves(s) == 1 && s.T <= (s.n_blocks <= 256 ? 8 : 2) * rows) return 1;
  const int64_t need = ((int64_t)s.T + rows - 1) / rows;
  return (int)(need < 1 ? 1 : need < kCus ? need : kCus);
}

struct BalanceWs : BalancePart {
  size_t bytes;
  BalanceWs(const meft_shape& s, void* ws) {
    Carver c(ws);
    const size_t g = balance_grid(s);
    prob = c.take<float>(g * s.n_blocks);
    count = c.take<int32_t>(g * s.n_blocks);
    lse2 = c.take<float>(g);
    tokens = c.take<int32_t>(g);
    dot = c.take<float>((s.n_blocks + 63) / 64);
    ticket = c.take<uint32_t>(1);
    bytes = c.off;
  }
};

#define MEFT_BALANCE_SHAPES(X)                                                     \
  if (s.n_blocks <= 64) X(1, 1);                                                   \
  else if (s.n_blocks <= 128) X(2, 1);                                             \
  else if (s.n_blocks <= 256) X(4, 1);                                             \
  else if (s.n_blocks <= 512) X(8, 1);                                             \
  else if (s.n_blocks <= 1024) X(16, 1);                                           \
  else if (s.n_blocks <= 2048) X(2, 16);                                           \
  else if (s.n_blocks <= 4096) X(4, 16);                                           \
  else if (s.n_blocks <= 8192) X(8, 16);                                           \
  else X(16, 16)
static_assert(kMaxBlocks <= 16 * 16 * 64, "balance_part_kernel and balance_grad_kernel hold a row in registers");

template <int Z, int W>
void launch_balance_part(const meft_shape& s, const float* scores, const int32_t* block_idx, const uint8_t* valid,
                         const BalancePart& part, const BalanceOut& out, hipStream_t st) {
  constexpr int rows = balance_rows(W, Z);
  const size_t lds = (size_t)s.n_blocks * 4 * (W == 1 ? rows + 1 : 1);
  if (W > 1) {
    static std::once_flag configured;   // up to 64 KB of counts beside the waves' values
    std::call_once(configured, [] {
      (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&balance_part_kernel<Z, W>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                kMaxBlocks * 4);
    });
  }
  MEFT_LAUNCH("balance_part", (balance_part_kernel<Z, W>), dim3(balance_grid(s)), dim3(balance_threads<Z, W>()), lds, st, scores,
              block_idx, valid, s.T, s.n_blocks, s.top_e, part, out);
}

bool balance_ok(const meft_balance* b) { return b && std::isfinite(b->balance) && std::isfinite(b->z); }

// ---- router gradient ------------------------------------------------------------------------
constexpr int kDwWgs = kCus;   // workgroups of dWg at most, where one of all tokens does not need more
// LDS of a workgroup of dh: its part of the router, in bytes
int dh_router_lds(const meft_shape& s) {
  const int all = s.dtype == MEFT_BF16 ? dh_steps<bf16_t>(s.n_blocks) * dh_step_bytes<bf16_t>()
                                       : dh_steps<float>(s.n_blocks) * dh_step_bytes<float>();
  return all < kDhLds ? all : kDhLds;
}
// workgroups of dh along the tokens: one for every compute unit beside dWg's, each with at least a tile per wave
int dh_along(const meft_shape& s, int slices) {
  const int64_t rounds = ((int64_t)s.T + 32 * kRgWaves - 1) / (32 * kRgWaves), most = (kCus + slices - 1) / slices;
  return (int)(rounds < most ? rounds : most);
}
struct RouteGradPlan {
  int slices, m, m_shift, groups, splits, per_split;
};
RouteGradPlan route_grad_plan(const meft_shape& s) {
  RouteGradPlan p{};
  p.slices = (s.d + kRgCols - 1) / kRgCols;
  p.m = s.n_blocks <= 32 ? 1 : 2;
  const int tiles = (s.n_blocks + 32 * p.m - 1) / (32 * p.m);
  while ((1 << p.m_shift) < tiles && (1 << p.m_shift) < kRgWaves) ++p.m_shift;
  const int m_waves = 1 << p.m_shift;
  p.groups = (tiles + m_waves - 1) / m_waves;
  // Splits of the tokens: what a wave's steps take, each split's partial sums on their way out and in, and the launch that adds
  // them, in us; at most a workgroup for every compute unit.  Whole call, us, splits of at least one step / by this: 256 tokens,
  // d 2048, 256 blocks 25.2 (16 splits) / 12.9 (1), 256 tokens, d 4096, 64 blocks 12.7 (4) / 8.3 (1); 2048 tokens, d 2048, 512 blocks 49.0 / 49.6.
  const double step_us = s.dtype == MEFT_BF16 ? 0.5 : 1.2 * p.m, part_us = 8.0 * s.n_blocks * (double)s.d / 5e6;
  int64_t want = (kDwWgs + p.slices * p.groups - 1) / (p.slices * p.groups);
  const int64_t steps = ((int64_t)s.T + 15) / 16;
  // Where a compute unit's 160 KB hold one workgroup only and dh takes up to half of them, dWg's are to run beside dh's and not
  // before: us, any number of splits / as many as that leaves, fp32, 747 tokens, d 1160, 294 blocks 44.5 / 35.0, 2000 tokens, d 1024,
  // 256 blocks 46.7 / 32.3; dh's workgroups in front instead 35.9 and 38.7.
  const int n_dh = dh_along(s, p.slices) * p.slices;
  if (2 * (dh_router_lds(s) + kDhDsLds) > 160 << 10 && n_dh <= kCus / 2) {
    const int64_t beside = (kCus - n_dh) / (p.slices * p.groups);
    want = beside < 1 ? 1 : beside;
  }
  const int k_waves = kRgWaves / m_waves;
  int64_t splits = 1;
  double best = 0;
  for (int64_t n = 1; n <= want && (n == 1 || n * k_waves <= steps); ++n) {
    const double us = (double)((steps + n * k_waves - 1) / (n * k_waves)) * step_us + (n > 1 ? n * part_us + 3.5 : 0);
    if (n == 1 || us < best) { best = us; splits = n; }
  }
  const int64_t per = (((int64_t)s.T + splits - 1) / splits + 15) / 16 * 16;
  p.per_split = (int)(per < 16 ? 16 : per);
  splits = ((int64_t)s.T + p.per_split - 1) / p.per_split;
  p.splits = (int)(splits < 1 ? 1 : splits);
  return p;
}

struct RouteGradWs {
  float *part, *part_bias;
  size_t bytes;
  RouteGradWs(const meft_shape& s, void* ws) {
    Carver c(ws);
    const RouteGradPlan p = route_grad_plan(s);
    part = c.take<float>(p.splits > 1 ? (size_t)p.splits * s.n_blocks * s.d : 0);
    part_bias = c.take<float>(p.splits > 1 ? (size_t)p.splits * s.n_blocks : 0);
    bytes = c.off;
  }
};

template <typename T, int M>
void launch_route_grad(const RouteGradArgs<T>& a, int wgs, int lds, hipStream_t st) {
  static std::once_flag configured;
  std::call_once(configured, [] {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&route_grad_kernel<T, M>), hipFuncAttributeMaxDynamicSharedMemorySize,
                              kDhLds + kDhDsLds);
  });
  MEFT_LAUNCH("route_grad", (route_grad_kernel<T, M>), dim3((unsigned)wgs), dim3(64 * kRgWaves), lds, st, a);
}

template <typename T>
meft_status route_bwd(const meft_shape& s, const void* h, const void* Wg, const float* ds, const void* add, void* dh, void* dWg,
                      float* dbias, void* ws, hipStream_t st) {
  const RouteGradPlan p = route_grad_plan(s);
  const RouteGradWs w(s, ws);
  const bool dw = dWg || dbias;
  const int dw_slices = dWg ? p.slices : 1, n_dw = dw ? dw_slices * p.groups * p.splits : 0;
  const int n_along = dh_along(s, p.slices), n_dh = dh ? n_along * p.slices : 0;
  if (n_dw + n_dh == 0) return MEFT_OK;
  const int w_lds = dh_router_lds(s), dh_lds = w_lds + kDhDsLds;
  const int dw_lds = p.m_shift == 2 ? 4 << 10 : 2 * p.m * 16 << 10;   // two of M * 64 x 64 sums, or the biases
  const int lds = dh && dh_lds > dw_lds ? dh_lds : dw_lds;
  const RouteGradArgs<T> a{static_cast<const T*>(h), static_cast<const T*>(Wg), static_cast<const T*>(add), ds, static_cast<T*>(dh),
                           static_cast<T*>(dWg), dbias, w.part, w.part_bias, s.T, s.d, s.n_blocks, p.m_shift, p.splits,
                           p.per_split, w_lds / 16, n_dw, dw_slices, n_along};
  if (p.m == 1) launch_route_grad<T, 1>(a, n_dw + n_dh, lds, st);
  else launch_route_grad<T, 2>(a, n_dw + n_dh, lds, st);
  if (dw && p.splits > 1) {
    const int64_t quads = dWg ? (int64_t)s.n_blocks * s.d / 4 : 0;
    MEFT_LAUNCH("route_dw_join", route_dw_join_kernel<T>, dim3((unsigned)((quads + 255) / 256 + 1)), dim3(256), 0, st, a);
  }
  return launch_status();
}

size_t block_workspace_bytes(const meft_shape& s) {
  size_t m = 256;
  for (const size_t b : {NormBwdWs(s, nullptr).bytes, BalanceWs(s, nullptr).bytes, RouteGradWs(s, nullptr).bytes})
    if (b > m) m = b;
  return m;
}

meft_status check_block_ws(const meft_shape& s, const void* ws, size_t have) {
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || have < block_workspace_bytes(s)) return MEFT_ERR_WORKSPACE;
  return MEFT_OK;
}

}  // namespace
}  // namespace meft

using namespace meft;

#define MEFT_BY_TYPE(f, ...) (s.dtype == MEFT_BF16 ? f<bf16_t>(__VA_ARGS__) : f<float>(__VA_ARGS__))

extern "C" {

size_t meft_block_workspace_bytes(const meft_shape* shape) {
  if (check_shape(shape) != MEFT_OK) return 0;
  return block_workspace_bytes(*shape);
}

meft_status meft_norm_fwd(const meft_shape* shape, const meft_norm* norm, const void* x, const void* gamma, const void* beta,
                          void* h, float* mean, float* rstd, void* stream) {
  const meft_status rc = check_shape(shape);
  if (rc != MEFT_OK) return rc;
  const meft_shape& s = *shape;
  if (!norm_ok(norm) || !ok16(x) || !ok16(gamma) || !null_or16(beta) || !ok16(h) || !aligned_as<float>(mean) || !aligned_as<float>(rstd))
    return MEFT_ERR_INVALID_ARG;
  if (s.T == 0) return MEFT_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  MEFT_API_LOCK();
  clear_stale_error();
  return MEFT_BY_TYPE(norm_fwd, s, *norm, kNormPlain, DropArgs{}, x, nullptr, gamma, beta, nullptr, h, mean, rstd, st);
}

meft_status meft_norm_bwd(const meft_shape* shape, const meft_norm* norm, const void* x, const void* gamma, const float* mean,
                          const float* rstd, const void* dh, const void* dy, void* dx, void* dgamma, void* dbeta, void* ws,
                          size_t ws_bytes, void* stream) {
  meft_status rc = check_shape(shape);
  if (rc != MEFT_OK) return rc;
  const meft_shape& s = *shape;
  if (!norm_ok(norm) || !ok16(x) || !ok16(gamma) || !rstd || !aligned_as<float>(rstd) || !ok16(dh) || !null_or16(dy) || !ok16(dx) ||
      !null_or16(dgamma) || !null_or16(dbeta) || (dbeta && !dgamma))
    return MEFT_ERR_INVALID_ARG;
  if (!aligned_as<float>(mean) || (norm->kind == MEFT_NORM_LAYER && !mean)) return MEFT_ERR_INVALID_ARG;
  if ((rc = check_block_ws(s, ws, ws_bytes)) != MEFT_OK) return rc;
  const size_t vec = row_bytes(s), rows = vec * s.T, stat = (size_t)s.T * 4, means = norm->kind == MEFT_NORM_LAYER ? stat : 0;
  if (!outputs_apart({{dx, rows}, {dgamma, vec}, {dbeta, vec}}, 1, {{x, rows}, {gamma, vec}, {mean, means}, {rstd, stat}}, {{dh, rows}, {dy, rows}}))
    return MEFT_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  MEFT_API_LOCK();
  clear_stale_error();
  return MEFT_BY_TYPE(norm_bwd, s, *norm, kNormPlain, DropArgs{}, x, gamma, mean, rstd, dh, dy, dx, nullptr, dgamma, dbeta, ws, st);
}

meft_status meft_dropout_add(const meft_shape* shape, const meft_drop* drop, const uint64_t* step, const void* out, const void* res,
                             void* y, void* stream) {
  const meft_status rc = check_shape(shape);
  if (rc != MEFT_OK) return rc;
  const meft_shape& s = *shape;
  const int thr = drop_threshold(drop);
  if (thr < 0 || !aligned_as<uint64_t>(step) || !ok16(out) || !null_or16(res) || !ok16(y)) return MEFT_ERR_INVALID_ARG;
  if (s.T == 0) return MEFT_OK;
  const int groups = s.d / 8;
  const int64_t spans = ((int64_t)s.T * groups + kDropSpan - 1) / kDropSpan, most = kDropWgs;
  const int64_t wgs = spans < most ? spans : most;
  const dim3 grid((unsigned)wgs);
  const uint32_t step_t = (uint32_t)(wgs * kDropSpan / groups), step_g = (uint32_t)(wgs * kDropSpan % groups);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const DropArgs a = drop_args(drop, step, thr);
  MEFT_API_LOCK();
  clear_stale_error();
#define DROPOUT(TY, DROP) MEFT_LAUNCH("dropout_add", (dropout_add_kernel<TY, DROP>), grid, dim3(256), 0, st, static_cast<const TY*>(out), \
                                     static_cast<const TY*>(res), static_cast<TY*>(y), s.T, groups, tile_div_inverse(groups), \
                                     step_t, step_g, past_l2(s), a)
  if (s.dtype == MEFT_BF16) {
    if (thr) DROPOUT(bf16_t, true);
    else DROPOUT(bf16_t, false);
  } else {
    if (thr) DROPOUT(float, true);
    else DROPOUT(float, false);
  }
#undef DROPOUT
  return launch_status();
}

meft_status meft_add_norm_fwd(const meft_shape* shape, const meft_norm* norm, const meft_drop* drop, const uint64_t* step,
                              const void* out, const void* res, const void* gamma, const void* beta, void* y, void* h, float* mean,
                              float* rstd, void* stream) {
  const meft_status rc = check_shape(shape);
  if (rc != MEFT_OK) return rc;
  const meft_shape& s = *shape;
  const int thr = drop_threshold(drop);
  if (!norm_ok(norm) || thr < 0 || !aligned_as<uint64_t>(step) || !ok16(out) || !ok16(res) || !ok16(gamma) || !null_or16(beta) ||
      !ok16(y) || !ok16(h) || y == h || !aligned_as<float>(mean) || !aligned_as<float>(rstd))
    return MEFT_ERR_INVALID_ARG;
  if (s.T == 0) return MEFT_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  MEFT_API_LOCK();
  clear_stale_error();
  return MEFT_BY_TYPE(norm_fwd, s, *norm, thr ? kNormDrop : kNormAdd, drop_args(drop, step, thr), res, out, gamma, beta, y, h, mean,
                      rstd, st);
}

meft_status meft_add_norm_bwd(const meft_shape* shape, const meft_norm* norm, const meft_drop* drop, const uint64_t* step,
                              const void* y, const void* gamma, const float* mean, const float* rstd, const void* dh, const void* dy,
                              void* dres, void* dout, void* dgamma, void* dbeta, void* ws, size_t ws_bytes, void* stream) {
  meft_status rc = check_shape(shape);
  if (rc != MEFT_OK) return rc;
  const meft_shape& s = *shape;
  const int thr = drop_threshold(drop);
  if (!norm_ok(norm) || thr < 0 || !aligned_as<uint64_t>(step) || !ok16(y) || !ok16(gamma) || !rstd || !aligned_as<float>(rstd) ||
      !ok16(dh) || !null_or16(dy) || !ok16(dres) || !ok16(dout) || dres == dout || !null_or16(dgamma) || !null_or16(dbeta) ||
      (dbeta && !dgamma))
    return MEFT_ERR_INVALID_ARG;
  if (!aligned_as<float>(mean) || (norm->kind == MEFT_NORM_LAYER && !mean)) return MEFT_ERR_INVALID_ARG;
  if ((rc = check_block_ws(s, ws, ws_bytes)) != MEFT_OK) return rc;
  const size_t vec = row_bytes(s), rows = vec * s.T, stat = (size_t)s.T * 4, means = norm->kind == MEFT_NORM_LAYER ? stat : 0;
  if (!outputs_apart({{dres, rows}, {dout, rows}, {dgamma, vec}, {dbeta, vec}}, 2, {{y, rows}, {gamma, vec}, {mean, means}, {rstd, stat}},
                     {{dh, rows}, {dy, rows}}))
    return MEFT_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  MEFT_API_LOCK();
  clear_stale_error();
  return MEFT_BY_TYPE(norm_bwd, s, *norm, thr ? kNormDrop : kNormAdd, drop_args(drop, step, thr), y, gamma, mean, rstd, dh, dy, dres,
                      dout, dgamma, dbeta, ws, st);
}

meft_status meft_balance_fwd(const meft_shape* shape, const meft_balance* balance, const float* scores, const int32_t* block_idx,
                             const uint8_t* valid, int32_t* counts, int32_t* n_valid, float* prob, float* loss, void* ws,
                             size_t ws_bytes, void* stream) {
  meft_status rc = check_shape(shape);
  if (rc != MEFT_OK) return rc;
  const meft_shape& s = *shape;
  if (!balance_ok(balance) || !ok16(scores) || !block_idx || !counts || !n_valid || !prob || !loss || !aligned_as<int32_t>(block_idx) ||
      !aligned_as<int32_t>(counts) || !aligned_as<int32_t>(n_valid) || !aligned_as<float>(prob) || !aligned_as<float>(loss))
    return MEFT_ERR_INVALID_ARG;
  if ((rc = check_block_ws(s, ws, ws_bytes)) != MEFT_OK) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const BalanceWs w(s, ws);
  const BalanceOut out{counts, n_valid, prob, loss, balance->balance, balance->z};
  MEFT_API_LOCK();
  clear_stale_error();
#define X(Z, W) launch_balance_part<Z, W>(s, scores, block_idx, valid, w, out, st)
  MEFT_BALANCE_SHAPES(X);
#undef X
  if (balance_waves(s) > 1 || balance_grid(s) > 1)
    MEFT_LAUNCH("balance_join", balance_join_kernel, dim3((s.n_blocks + 63) / 64), dim3(1024), 0, st, static_cast<const BalancePart&>(w),
                balance_grid(s), s.n_blocks, s.top_e, out);
  return launch_status();
}

meft_status meft_balance_bwd(const meft_shape* shape, const meft_balance* balance, const float* scores, const int32_t* counts,
                             const int32_t* n_valid, const uint8_t* valid, const float* dloss, float* dscores, void* stream) {
  const meft_status rc = check_shape(shape);
  if (rc != MEFT_OK) return rc;
  const meft_shape& s = *shape;
  if (!balance_ok(balance) || !ok16(scores) || !counts || !n_valid || !ok16(dscores) || !aligned_as<int32_t>(counts) ||
      !aligned_as<int32_t>(n_valid) || !aligned_as<float>(dloss))
    return MEFT_ERR_INVALID_ARG;
  if (s.T == 0) return MEFT_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int rows = balance_waves(s) == 1 ? 4 : 1;
  const int64_t need = ((int64_t)s.T + rows - 1) / rows, most = kCus * 8;
  const dim3 grid((unsigned)(need < most ? need : most));
  MEFT_API_LOCK();
  clear_stale_error();
#define X(Z, W)                                                                                                             \
  MEFT_LAUNCH("balance_grad", (balance_grad_kernel<Z, W>), grid, dim3(W == 1 ? 256 : 64 * W), 0, st, scores, counts, n_valid, valid, \
              dloss, s.T, s.n_blocks, s.top_e, balance->balance, balance->z, dscores)
  MEFT_BALANCE_SHAPES(X);
#undef X
  return launch_status();
}

meft_status meft_route_bwd(const meft_shape* shape, const void* h, const void* Wg, const float* dscores, const void* add, void* dh,
                           void* dWg, float* dbias, void* ws, size_t ws_bytes, void* stream) {
  meft_status rc = check_shape(shape);
  if (rc != MEFT_OK) return rc;
  const meft_shape& s = *shape;
  if (!ok16(h) || !ok16(Wg) || !ok16(dscores) || !null_or16(add) || !null_or16(dh) || !null_or16(dWg) || !aligned_as<float>(dbias) ||
      !(dh || dWg || dbias) || (add && !dh))
    return MEFT_ERR_INVALID_ARG;
  if ((rc = check_block_ws(s, ws, ws_bytes)) != MEFT_OK) return rc;
  const size_t rows = row_bytes(s) * s.T, router = row_bytes(s) * s.n_blocks, bias = (size_t)s.n_blocks * 4;
  if (!outputs_apart({{dh, rows}, {dWg, router}, {dbias, bias}}, 1, {{h, rows}, {Wg, router}, {dscores, bias * s.T}}, {{add, rows}}))
    return MEFT_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  MEFT_API_LOCK();
  clear_stale_error();
  return MEFT_BY_TYPE(route_bwd, s, h, Wg, dscores, add, dh, dWg, dbias, ws, st);
}

}  // extern "C"
