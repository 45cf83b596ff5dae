// A block's output joined to the residual stream, and the stream normalised
// for the next block, row by row:
//   u = post(z),  h = alpha x + act(gate) u,  y = pre(h),
// post and pre each nothing, a layer norm or an RMS norm; and the gradient:
//   e = dh + pre'(dy),  dx = alpha e,  dz = post'(act(gate) e),
//   dgate = act'(gate) sum e u over the rows that share a gate row.
#include <algorithm>

#include "elements.hpp"
#include "gba_device.hpp"
#include "gba_internal.hpp"
#include "row_place.hpp"

namespace gba {

typedef gba_residual_norm_args Args;

constexpr int kRowBlock = 256;
constexpr int kRowWaves = kRowBlock / kWave;
constexpr int kV = 4;                       // columns of a lane
constexpr int64_t kMaxRowGrid = 1 << 20;
constexpr int64_t kUnitBlocks = 512;        // most partial sums of the parameters' gradients

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

__device__ __forceinline__ float sigmoid(float a) { return 1.0f / (1.0f + expf(-a)); }

// Sums of two values over the block; every thread gets them.
__device__ __forceinline__ void block_sum2(float& a, float& b, float (*s)[kRowWaves]) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) {
    a += __shfl_xor(a, off, kWave);
    b += __shfl_xor(b, off, kWave);
  }
  const int w = threadIdx.x / kWave;
  __syncthreads();   // the last sums have been read
  if (lane_id() == 0) {
    s[0][w] = a;
    s[1][w] = b;
  }
  __syncthreads();
  a = b = 0.0f;
#pragma unroll
  for (int k = 0; k < kRowWaves; ++k) {
    a += s[0][k];
    b += s[1][k];
  }
}

// kV parameters of a norm, or what stands for those that are not there.
__device__ __forceinline__ void load_param(const void* p, int type, int64_t c, int count, float none, float (&o)[kV]) {
#pragma unroll
  for (int e = 0; e < kV; ++e) o[e] = none;
  if (p) load_part<kV>(p, type, c, count, o);
}
// The gate's factor in row r, and its derivative by the gate.
__device__ __forceinline__ void load_gate(const Args& a, int64_t r, int64_t c, int count, float (&f)[kV], float (&d)[kV]) {
#pragma unroll
  for (int e = 0; e < kV; ++e) f[e] = d[e] = 1.0f;
  if (a.gate_kind == GBA_GATE_NONE) return;
  load_part<kV>(a.gate, a.gate_type, r / a.gate_span * a.gate_stride + c, count, f);
  if (a.gate_kind != GBA_GATE_SIGMOID) return;
#pragma unroll
  for (int e = 0; e < kV; ++e) {
    f[e] = sigmoid(f[e]);
    d[e] = f[e] * (1.0f - f[e]);
  }
}

// How the rows are cut into units, the rows of a gate row (or all rows) in
// `cuts` equal parts: blocks take units in turn.
struct Units {
  int64_t span;      // rows of a gate row whose gradients are added up; else all rows
  int64_t cuts;      // units of it
  int64_t rows;      // of a unit
  int64_t units;
  bool gate;         // a gradient per gate row is added up
};
static Units units_of(const Args& a) {
  Units u;
  // (the same units, and so the same bits, with and without the gate's gradient)
  const bool shared = a.gate_kind != GBA_GATE_NONE && a.gate_span > 1;
  u.gate = shared && a.dgate;
  u.span = shared ? std::min(a.gate_span, a.n) : a.n;
  const int64_t G = ceil_div(a.n, u.span);
  u.cuts = std::min(u.span, std::max<int64_t>(1, kUnitBlocks / G));
  u.rows = ceil_div(u.span, u.cuts);
  u.cuts = ceil_div(u.span, u.rows);
  u.units = G * u.cuts;
  return u;
}

// --------------------------------------------- rows read from memory again
template <typename TS, typename TZ>
__global__ void __launch_bounds__(kRowBlock)
residual_norm_wide_kernel(Args a) {
  __shared__ float s_sum[2][kRowWaves];
  const float D = (float)a.D, eps = (float)a.eps, alpha = (float)a.alpha;
  for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x) {
    const TS* x = static_cast<const TS*>(a.x) + r * a.x_stride;
    const TZ* z = static_cast<const TZ*>(a.z) + r * a.z_stride;
    TS* h = static_cast<TS*>(a.h) + r * a.h_stride;
    float mean = 0.0f, rstd = 1.0f, unused = 0.0f;
    if (a.post != GBA_ROW_NORM_NONE) {
      if (a.post == GBA_ROW_NORM_LAYER) {
        for (int c = threadIdx.x * kV; c < a.D; c += kRowBlock * kV) {
          float v[kV];
          load_part<TZ, kV>(z + c, a.D - c, v);
#pragma unroll
          for (int e = 0; e < kV; ++e) mean += v[e];
        }
        block_sum2(mean, unused, s_sum);
        mean /= D;
      }
      float sq = 0.0f;
      for (int c = threadIdx.x * kV; c < a.D; c += kRowBlock * kV) {
        float v[kV];
        load_part<TZ, kV>(z + c, a.D - c, v);
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          const float d = c + e < a.D ? v[e] - mean : 0.0f;
          sq = __builtin_fmaf(d, d, sq);
        }
      }
      block_sum2(sq, unused, s_sum);
      rstd = 1.0f / sqrtf(sq / D + eps);
      if (threadIdx.x == 0) {
        if (a.post_mean) a.post_mean[r] = mean;
        if (a.post_rstd) a.post_rstd[r] = rstd;
      }
    }
    float sum = 0.0f;
    for (int c = threadIdx.x * kV; c < a.D; c += kRowBlock * kV) {
      const int count = a.D - c;
      float v[kV], u[kV], w[kV], b[kV], f[kV], d[kV];
      load_part<TS, kV>(x + c, count, v);
      load_part<TZ, kV>(z + c, count, u);
      load_param(a.post_weight, a.weight_type, c, count, 1.0f, w);
      load_param(a.post_bias, a.weight_type, c, count, 0.0f, b);
      load_gate(a, r, c, count, f, d);
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        v[e] = __builtin_fmaf(f[e], __builtin_fmaf((u[e] - mean) * rstd, w[e], b[e]), alpha * v[e]);
        if (c + e < a.D) sum += (float)(TS)v[e];
      }
      store_part<TS, kV>(h + c, count, v);
    }
    if (a.pre == GBA_ROW_NORM_NONE) continue;
    mean = 0.0f;
    if (a.pre == GBA_ROW_NORM_LAYER) {
      block_sum2(sum, unused, s_sum);
      mean = sum / D;
    }
    float sq = 0.0f;   // (a thread reads again what it has written itself)
    for (int c = threadIdx.x * kV; c < a.D; c += kRowBlock * kV) {
      float v[kV];
      load_part<TS, kV>(h + c, a.D - c, v);
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const float d = c + e < a.D ? v[e] - mean : 0.0f;
        sq = __builtin_fmaf(d, d, sq);
      }
    }
    block_sum2(sq, unused, s_sum);
    rstd = 1.0f / sqrtf(sq / D + eps);
    if (threadIdx.x == 0) {
      if (a.pre_mean) a.pre_mean[r] = mean;
      if (a.pre_rstd) a.pre_rstd[r] = rstd;
    }
    TZ* y = static_cast<TZ*>(a.y) + r * a.y_stride;
    for (int c = threadIdx.x * kV; c < a.D; c += kRowBlock * kV) {
      const int count = a.D - c;
      float v[kV], w[kV], b[kV];
      load_part<TS, kV>(h + c, count, v);
      load_param(a.pre_weight, a.weight_type, c, count, 1.0f, w);
      load_param(a.pre_bias, a.weight_type, c, count, 0.0f, b);
#pragma unroll
      for (int e = 0; e < kV; ++e) v[e] = __builtin_fmaf((v[e] - mean) * rstd, w[e], b[e]);
      store_part<TZ, kV>(y + c, count, v);
    }
  }
}

// What the gradient of kV elements of a row is made of.
struct RowBack {
  float xh[kV], hh[kV];    // of the norm before: what was normalised, and dy by its weight
  float zh[kV], wz[kV];    // of the norm after the block, and its weight
  float u[kV];             // what the gate multiplies
  float f[kV], df[kV];     // the gate's factor and derivative
  float dy[kV], dh[kV];
};
struct RowStat {
  float mean_h, rstd_h, mean_z, rstd_z;
};
__device__ __forceinline__ RowStat row_stat(const Args& a, int64_t r) {
  RowStat s{0.0f, 1.0f, 0.0f, 1.0f};
  if (a.pre != GBA_ROW_NORM_NONE) s.rstd_h = a.pre_rstd[r];
  if (a.pre == GBA_ROW_NORM_LAYER) s.mean_h = a.pre_mean[r];
  if (a.post != GBA_ROW_NORM_NONE) s.rstd_z = a.post_rstd[r];
  if (a.post == GBA_ROW_NORM_LAYER) s.mean_z = a.post_mean[r];
  return s;
}
template <typename TS, typename TZ>
__device__ __forceinline__ void load_back(const Args& a, int64_t r, int c, const RowStat& s, bool after, RowBack& o) {
  const int count = a.D - c;
  float v[kV], w[kV], b[kV];
#pragma unroll
  for (int e = 0; e < kV; ++e) o.xh[e] = o.hh[e] = o.dy[e] = o.dh[e] = 0.0f;
  if (a.pre != GBA_ROW_NORM_NONE) {
    load_part<TS, kV>(static_cast<const TS*>(a.h) + r * a.h_stride + c, count, v);
    load_part<TZ, kV>(static_cast<const TZ*>(a.dy) + r * a.dy_stride + c, count, o.dy);
    load_param(a.pre_weight, a.weight_type, c, count, 1.0f, w);
#pragma unroll
    for (int e = 0; e < kV; ++e) {
      o.xh[e] = (v[e] - s.mean_h) * s.rstd_h;
      o.hh[e] = o.dy[e] * w[e];
    }
  }
  if (!after) return;
  if (a.dh) load_part<TS, kV>(static_cast<const TS*>(a.dh) + r * a.dh_stride + c, count, o.dh);
  load_part<TZ, kV>(static_cast<const TZ*>(a.z) + r * a.z_stride + c, count, v);
  load_param(a.post_weight, a.weight_type, c, count, 1.0f, o.wz);
  load_param(a.post_bias, a.weight_type, c, count, 0.0f, b);
  load_gate(a, r, c, count, o.f, o.df);
#pragma unroll
  for (int e = 0; e < kV; ++e) {
    o.zh[e] = (v[e] - s.mean_z) * s.rstd_z;
    o.u[e] = __builtin_fmaf(o.zh[e], o.wz[e], b[e]);
  }
}
// The gradient of h's element e: m1 and m2 are the means of hh (layer norm) and of hh * xh.
__device__ __forceinline__ float stream_grad(const RowBack& b, int e, const RowStat& s, float m1, float m2) {
  return b.dh[e] + s.rstd_h * (b.hh[e] - m1 - b.xh[e] * m2);
}

// A row's four means: of hh, of hh * xh, and the same of the norm after the block.
template <typename TS, typename TZ>
__global__ void __launch_bounds__(kRowBlock)
residual_norm_means_kernel(Args a, float* __restrict__ means) {
  __shared__ float s_sum[2][kRowWaves];
  const float D = (float)a.D;
  for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x) {
    const RowStat st = row_stat(a, r);
    float m[4] = {};
    RowBack b;
    if (a.pre != GBA_ROW_NORM_NONE) {
      for (int c = threadIdx.x * kV; c < a.D; c += kRowBlock * kV) {
        load_back<TS, TZ>(a, r, c, st, false, b);
#pragma unroll
        for (int e = 0; e < kV; ++e) {   // (past the row's end dy is 0)
          m[0] += b.hh[e];
          m[1] = __builtin_fmaf(b.hh[e], b.xh[e], m[1]);
        }
      }
      block_sum2(m[0], m[1], s_sum);
      m[0] = a.pre == GBA_ROW_NORM_LAYER ? m[0] / D : 0.0f;
      m[1] /= D;
    }
    if (a.post != GBA_ROW_NORM_NONE) {
      for (int c = threadIdx.x * kV; c < a.D; c += kRowBlock * kV) {
        load_back<TS, TZ>(a, r, c, st, true, b);
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          const float k = c + e < a.D ? stream_grad(b, e, st, m[0], m[1]) * b.f[e] * b.wz[e] : 0.0f;
          m[2] += k;
          m[3] = __builtin_fmaf(k, b.zh[e], m[3]);
        }
      }
      block_sum2(m[2], m[3], s_sum);
      m[2] = a.post == GBA_ROW_NORM_LAYER ? m[2] / D : 0.0f;
      m[3] /= D;
    }
    if (threadIdx.x < 4) means[r * 4 + threadIdx.x] = m[threadIdx.x];
  }
}

template <typename TS, typename TZ>
__global__ void __launch_bounds__(kRowBlock)
residual_norm_rows_kernel(Args a, const float* __restrict__ means) {
  const float alpha = (float)a.alpha;
  for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x) {
    const RowStat st = row_stat(a, r);
    float m[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) m[k] = means[r * 4 + k];
    for (int c = threadIdx.x * kV; c < a.D; c += kRowBlock * kV) {
      const int count = a.D - c;
      RowBack b;
      load_back<TS, TZ>(a, r, c, st, true, b);
      float dx[kV], dz[kV], dg[kV];
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const float g = stream_grad(b, e, st, m[0], m[1]);
        dx[e] = alpha * g;
        dg[e] = g * b.u[e] * b.df[e];
        const float k = g * b.f[e];
        dz[e] = a.post == GBA_ROW_NORM_NONE ? k : st.rstd_z * (k * b.wz[e] - m[2] - b.zh[e] * m[3]);
      }
      if (a.dx) store_part<TS, kV>(static_cast<TS*>(a.dx) + r * a.dx_stride + c, count, dx);
      if (a.dz) store_part<TZ, kV>(static_cast<TZ*>(a.dz) + r * a.dz_stride + c, count, dz);
      if (a.dgate && a.gate_span == 1) store_part<kV>(a.dgate, a.gate_type, r * a.dgate_stride + c, count, dg);
    }
  }
}

// Partial sums over units of rows: of the four parameters' gradients over all
// units of a block, of the gate's over each unit.  A wave per slice of
// columns, four waves' sums joined in LDS.
template <typename TS, typename TZ>
__global__ void __launch_bounds__(kRowBlock)
residual_norm_columns_kernel(Args a, const float* __restrict__ means, Units un, float* __restrict__ partial,
                             float* __restrict__ gate_partial) {
  __shared__ float s_part[kRowWaves][kWave * kV];
  const int w = threadIdx.x / kWave, lane = lane_id();
  const int c = (int)blockIdx.y * (kWave * kV) + lane * kV;
  float sum[4][kV] = {};
  // adds up `v` over the waves and hands each column's sum to `to`
  auto join = [&](float (&v)[kV], auto to) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kV; ++e) s_part[w][lane * kV + e] = v[e];
    __syncthreads();
    const int64_t cc = (int64_t)blockIdx.y * (kWave * kV) + threadIdx.x;
    float t = 0.0f;
#pragma unroll
    for (int k = 0; k < kRowWaves; ++k) t += s_part[k][threadIdx.x];
    if (cc < a.D) to(cc, t);
  };
  static_assert(kRowBlock == kWave * kV, "a thread per column of the slice");
  for (int64_t u = blockIdx.x; u < un.units; u += gridDim.x) {
    const int64_t g = u / un.cuts, first = g * un.span + (u % un.cuts) * un.rows;
    int64_t end = first + un.rows;
    end = end < (g + 1) * un.span ? end : (g + 1) * un.span;
    end = end < a.n ? end : a.n;
    float dg[kV] = {};
    if (c < a.D) {
      for (int64_t r = first + w; r < end; r += kRowWaves) {
        const RowStat st = row_stat(a, r);
        RowBack b;
        load_back<TS, TZ>(a, r, c, st, true, b);
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          const float gr = stream_grad(b, e, st, means[r * 4], means[r * 4 + 1]);
          dg[e] += gr * b.u[e] * b.df[e];
          const float k = gr * b.f[e];
          sum[0][e] = __builtin_fmaf(k, b.zh[e], sum[0][e]);
          sum[1][e] += k;
          sum[2][e] = __builtin_fmaf(b.dy[e], b.xh[e], sum[2][e]);
          sum[3][e] += b.dy[e];
        }
      }
    }
    if (un.gate)
      join(dg, [&](int64_t cc, float t) {
        const float v[1] = {t};
        if (un.cuts == 1) store_part<1>(a.dgate, a.gate_type, g * a.dgate_stride + cc, 1, v);
        else gate_partial[u * a.D + cc] = t;
      });
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    join(sum[k], [&](int64_t cc, float t) { partial[((int64_t)blockIdx.x * 4 + k) * a.D + cc] = t; });
}

// ------------------------------------------------------ rows in registers
constexpr int kRegBlock = 512;
constexpr int kWidest = 1024;             // most threads of a row
constexpr int kRegElements = 8;           // of a row, a thread's most
constexpr int kRegColumns = kWidest * kRegElements;
constexpr int64_t kRegBlocks = 2048;      // most blocks of a forward call

template <typename TZ, int LPR, int NV>
struct NormShape {
  static constexpr int V = kVec<TZ>;
  static constexpr int E = V * NV;
  static constexpr int BLOCK = LPR > kRegBlock ? LPR : kRegBlock;
  static constexpr int G = BLOCK / LPR;         // rows of a block at a time
  static constexpr int WAVES = BLOCK / kWave;
};

// A norm's parameters, or what stands for those that are not there.
template <typename At, int NV, int V>
__device__ __forceinline__ void load_params(const At& at, const void* p, int type, float none, float (&o)[NV][V]) {
#pragma unroll
  for (int k = 0; k < NV; ++k) {
#pragma unroll
    for (int e = 0; e < V; ++e) o[k][e] = none;
    if (p) at.load(p, type, k, o[k]);
  }
}
// The gate's row g as it is.
template <typename At, int NV, int V>
__device__ __forceinline__ void load_gate_row(const At& at, const Args& a, int64_t g, float (&o)[NV][V]) {
  const int64_t from = g * a.gate_stride;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (a.gate_type == GBA_F32) at.load(static_cast<const float*>(a.gate) + from, k, o[k]);
    else if (a.gate_type == GBA_BF16) at.load(static_cast<const bf16_t*>(a.gate) + from, k, o[k]);
    else at.load(static_cast<const f16_t*>(a.gate) + from, k, o[k]);
  }
}
template <int NV, int V>
__device__ __forceinline__ void gate_factors(const Args& a, float (&f)[NV][V]) {
  if (a.gate_kind != GBA_GATE_SIGMOID) return;
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < V; ++e) f[k][e] = sigmoid(f[k][e]);
}

// The mean (layer norm) and the reciprocal root of a row's norm, from registers.
template <int LPR, int WAVES, typename At, int NV, int V>
__device__ __forceinline__ void row_stats(const At& at, int kind, float D, float eps, const float (&v)[NV][V],
                                          float (*s)[1][WAVES], int& buffer, float& mean, float& rstd) {
  float t[1] = {0.0f};
  mean = 0.0f;
  if (kind == GBA_ROW_NORM_LAYER) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) t[0] += at.own(k, e) ? v[k][e] : 0.0f;
    row_sum<LPR, WAVES>(t, s, buffer);
    mean = t[0] / D;
    t[0] = 0.0f;
  }
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = at.own(k, e) ? v[k][e] - mean : 0.0f;
      t[0] = __builtin_fmaf(d, d, t[0]);
    }
  row_sum<LPR, WAVES>(t, s, buffer);
  rstd = 1.0f / sqrtf(t[0] / D + eps);
}

template <typename TS, typename TZ, int LPR, int NV>
__global__ void __launch_bounds__((NormShape<TZ, LPR, NV>::BLOCK), 4)
residual_norm_kernel(Args a, int64_t per, uint32_t span) {
  typedef NormShape<TZ, LPR, NV> S;
  constexpr int V = S::V;
  typedef typename VecOf<TS, V>::type stream_vec;
  typedef typename VecOf<TZ, V>::type vec;
  __shared__ float s_sum[2][1][S::WAVES];
  const int gl = threadIdx.x % LPR, grp = threadIdx.x / LPR;
  const RowPlace<V, LPR, NV> at(gl, a.D);
  const float D = (float)a.D, eps = (float)a.eps, alpha = (float)a.alpha;
  float wz[NV][V], bz[NV][V], wh[NV][V], bh[NV][V], f[NV][V], fn[NV][V];
  load_params(at, a.post_weight, a.weight_type, 1.0f, wz);
  load_params(at, a.post_bias, a.weight_type, 0.0f, bz);
  load_params(at, a.pre_weight, a.weight_type, 1.0f, wh);
  load_params(at, a.pre_bias, a.weight_type, 0.0f, bh);
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < V; ++e) f[k][e] = fn[k][e] = 1.0f;
  const bool gated = a.gate_kind != GBA_GATE_NONE, each = gated && span == 1;
  int64_t gate_row = -1;
  const int64_t r0 = (int64_t)blockIdx.x * per, r1 = r0 + per < a.n ? r0 + per : a.n;
  stream_vec x[NV], xn[NV];
  vec z[NV], zn[NV];
  auto load_row = [&](int64_t rb, stream_vec (&xv)[NV], vec (&zv)[NV], float (&g)[NV][V]) {
    const int64_t r = rb + grp < r1 ? rb + grp : r1 - 1;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      xv[k] = at.load_raw(static_cast<const TS*>(a.x) + r * a.x_stride, k);
      zv[k] = at.load_raw(static_cast<const TZ*>(a.z) + r * a.z_stride, k);
    }
    if (each) load_gate_row(at, a, r, g);
  };
  int buffer = 0;
  if (r0 < r1) load_row(r0, x, z, fn);
  for (int64_t rb = r0; rb < r1; rb += S::G) {
    const int64_t r = rb + grp;
    const bool active = r < r1;
    if (each) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) f[k][e] = fn[k][e];
      gate_factors(a, f);
    } else if (gated) {
      const int64_t g = (uint32_t)(active ? r : r1 - 1) / span;
      if (g != gate_row) {
        gate_row = g;
        load_gate_row(at, a, g, f);
        gate_factors(a, f);
      }
    }
    if (rb + S::G < r1) load_row(rb + S::G, xn, zn, fn);
    float v[NV][V], mean = 0.0f, rstd = 1.0f, pre_mean = 0.0f, pre_rstd = 1.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) v[k][e] = (float)z[k][e];
    if (a.post != GBA_ROW_NORM_NONE) row_stats<LPR, S::WAVES>(at, a.post, D, eps, v, s_sum, buffer, mean, rstd);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        v[k][e] = __builtin_fmaf(f[k][e], __builtin_fmaf((v[k][e] - mean) * rstd, wz[k][e], bz[k][e]),
                                 alpha * (float)x[k][e]);
        v[k][e] = (float)(TS)v[k][e];   // what pre normalises is the stream as it is stored
      }
    if (a.pre != GBA_ROW_NORM_NONE) row_stats<LPR, S::WAVES>(at, a.pre, D, eps, v, s_sum, buffer, pre_mean, pre_rstd);
    else if (LPR > kWave && a.post == GBA_ROW_NORM_NONE) __syncthreads();   // h may be x, and rows' last vectors overlap
    if (active) {
      if (gl == 0) {
        if (a.post_mean) a.post_mean[r] = mean;
        if (a.post_rstd) a.post_rstd[r] = rstd;
        if (a.pre_mean) a.pre_mean[r] = pre_mean;
        if (a.pre_rstd) a.pre_rstd[r] = pre_rstd;
      }
      TS* h = static_cast<TS*>(a.h) + r * a.h_stride;
      TZ* y = static_cast<TZ*>(a.y) + r * a.y_stride;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        at.store(h, k, v[k]);
        if (a.pre == GBA_ROW_NORM_NONE) continue;
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = __builtin_fmaf((v[k][e] - pre_mean) * pre_rstd, wh[k][e], bh[k][e]);
        at.store(y, k, o);
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      x[k] = xn[k];
      z[k] = zn[k];
    }
  }
}

// Where a block is in its units: at rows rb .. of unit u, whose last is end - 1.
struct UnitCursor {
  int64_t u, g, rb, end;
  __device__ __forceinline__ void enter(const Units& un, int64_t n) {
    g = u / un.cuts;
    rb = g * un.span + (u % un.cuts) * un.rows;
    end = rb + un.rows;
    end = end < (g + 1) * un.span ? end : (g + 1) * un.span;
    end = end < n ? end : n;
  }
};

// SHARED: the gate's gradient is added up over the rows of a unit.
template <typename TS, typename TZ, int LPR, int NV, bool SHARED>
__global__ void __launch_bounds__((NormShape<TZ, LPR, NV>::BLOCK), 2)
residual_norm_grad_kernel(Args a, Units un, float* __restrict__ partial, float* __restrict__ gate_partial) {
  typedef NormShape<TZ, LPR, NV> S;
  constexpr int V = S::V;
  constexpr int TEAM = LPR < kWave ? kWave : LPR;
  constexpr int TEAMS = S::BLOCK / TEAM;
  constexpr int COLS = LPR * S::E;
  typedef typename VecOf<TS, V>::type stream_vec;
  typedef typename VecOf<TZ, V>::type vec;
  __shared__ float s_sum[2][2][S::WAVES];
  __shared__ float s_part[TEAMS > 1 ? TEAMS * COLS : 1];
  const int gl = threadIdx.x % LPR, grp = threadIdx.x / LPR;
  const RowPlace<V, LPR, NV> at(gl, a.D);
  const float D = (float)a.D, alpha = (float)a.alpha;
  const bool pre = a.pre != GBA_ROW_NORM_NONE, post = a.post != GBA_ROW_NORM_NONE;
  const bool gated = a.gate_kind != GBA_GATE_NONE, each = gated && a.gate_span == 1;
  float wz[NV][V], bz[NV][V], wh[NV][V], f[NV][V], fn[NV][V];
  float sum[4][NV][V], dg[NV][V];
  load_params(at, a.post_weight, a.weight_type, 1.0f, wz);
  load_params(at, a.post_bias, a.weight_type, 0.0f, bz);
  load_params(at, a.pre_weight, a.weight_type, 1.0f, wh);
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      f[k][e] = fn[k][e] = 1.0f;
      dg[k][e] = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i][k][e] = 0.0f;
    }
  stream_vec h[NV] = {}, dh[NV] = {}, hn[NV] = {}, dhn[NV] = {};
  vec z[NV] = {}, dy[NV] = {}, zn[NV] = {}, dyn[NV] = {};
  RowStat st, stn;
  auto load_row = [&](const UnitCursor& c, stream_vec (&hv)[NV], stream_vec (&dhv)[NV], vec (&zv)[NV], vec (&dyv)[NV],
                      RowStat& s, float (&g)[NV][V]) {
    const int64_t r = c.rb + grp < c.end ? c.rb + grp : c.end - 1;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      zv[k] = at.load_raw(static_cast<const TZ*>(a.z) + r * a.z_stride, k);
      if (pre) {
        hv[k] = at.load_raw(static_cast<const TS*>(a.h) + r * a.h_stride, k);
        dyv[k] = at.load_raw(static_cast<const TZ*>(a.dy) + r * a.dy_stride, k);
      }
      if (a.dh) dhv[k] = at.load_raw(static_cast<const TS*>(a.dh) + r * a.dh_stride, k);
    }
    s = row_stat(a, r);
    if (each) load_gate_row(at, a, r, g);
  };
  // adds `v` up over the block's rows and hands each column's sum to `to`
  auto join = [&](float (&v)[NV][V], auto to) {
    if constexpr (LPR < kWave) {
#pragma unroll
      for (int off = LPR; off < kWave; off <<= 1)
#pragma unroll
        for (int e = 0; e < V; ++e) v[0][e] += __shfl_xor(v[0][e], off, kWave);   // (NV is 1)
    }
    if constexpr (TEAMS > 1) {
      __syncthreads();   // the last sums have been read
      if ((int)(threadIdx.x % TEAM) < LPR) {
        float* s = s_part + threadIdx.x / TEAM * COLS;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (at.own(k, e)) s[at.col[k] + e] = v[k][e];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < a.D; c += S::BLOCK) {
        float t = 0.0f;
#pragma unroll
        for (int m = 0; m < TEAMS; ++m) t += s_part[m * COLS + c];
        to(c, t);
      }
    } else {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (at.own(k, e)) to(at.col[k] + e, v[k][e]);
    }
  };
  UnitCursor now{(int64_t)blockIdx.x, 0, 0, 0};
  now.enter(un, a.n);
  load_row(now, h, dh, z, dy, st, fn);
  bool entered = true;
  int buffer = 0;
  for (;;) {
    UnitCursor next = now;
    next.rb += S::G;
    const bool leaves = next.rb >= now.end;
    if (leaves) {
      next.u += gridDim.x;
      if (next.u < un.units) next.enter(un, a.n);
    }
    const bool more = next.u < un.units;
    if (each) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) f[k][e] = fn[k][e];
      gate_factors(a, f);
    } else if (gated && entered) {
      load_gate_row(at, a, now.g, f);
      gate_factors(a, f);
    }
    if (more) load_row(next, hn, dhn, zn, dyn, stn, fn);
    const int64_t r = now.rb + grp;
    const bool active = r < now.end;
    float xh[NV][V], e_[NV][V], t[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        xh[k][e] = ((float)h[k][e] - st.mean_h) * st.rstd_h;
        const float g = active && at.own(k, e) ? (float)dy[k][e] : 0.0f;
        e_[k][e] = g * wh[k][e];
        t[0] += e_[k][e];
        t[1] = __builtin_fmaf(e_[k][e], xh[k][e], t[1]);
        sum[2][k][e] = __builtin_fmaf(g, xh[k][e], sum[2][k][e]);
        sum[3][k][e] += g;
      }
    if (pre) {
      row_sum<LPR, S::WAVES>(t, s_sum, buffer);
      const float m1 = a.pre == GBA_ROW_NORM_LAYER ? t[0] / D : 0.0f, m2 = t[1] / D;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          // (a foreign element's dy counts here: its column's owner stores the same)
          const float hh = (float)dy[k][e] * wh[k][e];
          e_[k][e] = (float)dh[k][e] + st.rstd_h * (hh - m1 - xh[k][e] * m2);
        }
    } else {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) e_[k][e] = (float)dh[k][e];
    }
    // from here xh is the normalised output of the block
    float kk[NV][V], dgate[NV][V];
    t[0] = t[1] = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const bool own = active && at.own(k, e);
        xh[k][e] = ((float)z[k][e] - st.mean_z) * st.rstd_z;
        const float u = __builtin_fmaf(xh[k][e], wz[k][e], bz[k][e]);
        dgate[k][e] = e_[k][e] * u;
        if (SHARED) dg[k][e] += own ? dgate[k][e] : 0.0f;
        const float g = e_[k][e] * f[k][e];
        sum[0][k][e] += own ? g * xh[k][e] : 0.0f;
        sum[1][k][e] += own ? g : 0.0f;
        kk[k][e] = g * wz[k][e];
        t[0] += own ? kk[k][e] : 0.0f;
        t[1] += own ? kk[k][e] * xh[k][e] : 0.0f;
      }
    if (post) {
      row_sum<LPR, S::WAVES>(t, s_sum, buffer);
      const float m1 = a.post == GBA_ROW_NORM_LAYER ? t[0] / D : 0.0f, m2 = t[1] / D;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) kk[k][e] = st.rstd_z * (kk[k][e] - m1 - xh[k][e] * m2);
    } else if (LPR > kWave && !pre) {
      __syncthreads();   // dx may be dh, dz dy, and rows' last vectors overlap
    }
    if (active) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = alpha * e_[k][e];
        if (a.dx) at.store(static_cast<TS*>(a.dx) + r * a.dx_stride, k, o);
        if (a.dz) at.store(static_cast<TZ*>(a.dz) + r * a.dz_stride, k, kk[k]);
        if (!SHARED && each && a.dgate) {
#pragma unroll
          for (int e = 0; e < V; ++e)
            o[e] = dgate[k][e] * (a.gate_kind == GBA_GATE_SIGMOID ? f[k][e] * (1.0f - f[k][e]) : 1.0f);
          const int64_t to = r * a.dgate_stride;
          if (a.gate_type == GBA_F32) at.store(static_cast<float*>(a.dgate) + to, k, o);
          else if (a.gate_type == GBA_BF16) at.store(static_cast<bf16_t*>(a.dgate) + to, k, o);
          else at.store(static_cast<f16_t*>(a.dgate) + to, k, o);
        }
      }
    }
    if (SHARED && leaves) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (a.gate_kind == GBA_GATE_SIGMOID) dg[k][e] *= f[k][e] * (1.0f - f[k][e]);
      join(dg, [&](int c, float v) {
        const float o[1] = {v};
        if (un.cuts == 1) store_part<1>(a.dgate, a.gate_type, now.g * a.dgate_stride + c, 1, o);
        else gate_partial[now.u * a.D + c] = v;
      });
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) dg[k][e] = 0.0f;
    }
    if (!more) break;
    now = next;
    entered = leaves;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      h[k] = hn[k];
      dh[k] = dhn[k];
      z[k] = zn[k];
      dy[k] = dyn[k];
    }
    st = stn;
  }
  void* const outs[4] = {a.dpost_weight, a.dpost_bias, a.dpre_weight, a.dpre_bias};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (!outs[i]) continue;
    join(sum[i], [&](int c, float v) {
      const float o[1] = {v};
      if (gridDim.x == 1) store_part<1>(outs[i], a.grad_type, c, 1, o);   // the only block writes the sums themselves
      else partial[((int64_t)blockIdx.x * 4 + i) * a.D + c] = v;
    });
  }
}

// The parameters' gradients from the blocks' partial sums, and the gate's from
// the units': 64 columns a block, each wave a share of the sums.
constexpr int kJoinBlock = 1024;
constexpr int kJoinWaves = kJoinBlock / kWave;
__global__ void __launch_bounds__(kJoinBlock)
residual_norm_join_kernel(Args a, const float* __restrict__ partial, int64_t parts, Units un,
                          const float* __restrict__ gate_partial) {
  __shared__ float s_sum[kJoinWaves][kWave];
  const int w = threadIdx.x / kWave, lane = lane_id();
  const int64_t c = (int64_t)blockIdx.x * kWave + lane;
  const int which = (int)blockIdx.y;   // a parameter, or 4 + a gate row
  void* const out = which == 0 ? a.dpost_weight : which == 1 ? a.dpost_bias : which == 2 ? a.dpre_weight : a.dpre_bias;
  if (which < 4 && !out) return;
  const float* from = which < 4 ? partial + which * (int64_t)a.D : gate_partial + (int64_t)(which - 4) * un.cuts * a.D;
  const int64_t count = which < 4 ? parts : un.cuts, step = which < 4 ? 4 * (int64_t)a.D : a.D;
  float s[1] = {0.0f};
  if (c < a.D) {
#pragma unroll 8
    for (int64_t p = w; p < count; p += kJoinWaves) s[0] += from[p * step + c];
  }
  s_sum[w][lane] = s[0];
  __syncthreads();
  if (w != 0 || c >= a.D) return;
  s[0] = 0.0f;
#pragma unroll
  for (int k = 0; k < kJoinWaves; ++k) s[0] += s_sum[k][lane];
  if (which >= 4) {
    store_part<1>(a.dgate, a.gate_type, (which - 4) * a.dgate_stride + c, 1, s);
    return;
  }
  store_part<1>(out, a.grad_type, c, 1, s);
}

// ------------------------------------------------------------- launching
// Scratch: partial sums of the parameters' gradients (a row of four per block)
// and of the gate's (a row per unit), and a row's means.
struct NormRoom {
  size_t partial, gate, means, bytes;
};
static NormRoom norm_room(int64_t n, int32_t D) {
  NormRoom r;
  // (units: at most as many as rows of whole gate rows, below 2 n; fewer than 2 kUnitBlocks where they are joined)
  r.partial = 0;
  r.gate = align_up((size_t)std::min(2 * n, kUnitBlocks) * 4 * D * sizeof(float));
  r.means = r.gate + align_up((size_t)std::min(2 * n, 2 * kUnitBlocks) * D * sizeof(float));
  r.bytes = r.means + align_up((size_t)n * 4 * sizeof(float)) + 256;
  return r;
}
size_t residual_norm_grad_workspace_bytes(int64_t n, int32_t D) { return norm_room(n, D).bytes; }

// Calls f.run<LPR, NV>() for the shape of rows of D columns: as few threads as
// hold the row, one vector each up to a wave, then as many as kRegElements allow.
template <typename TZ, typename F>
static hipError_t with_shape(int32_t D, const F& f) {
  const int vecs = (int)ceil_div(D, kVec<TZ>);
  if (vecs <= 1) return f.template run<1, 1>();
  if (vecs <= 2) return f.template run<2, 1>();
  if (vecs <= 4) return f.template run<4, 1>();
  if (vecs <= 8) return f.template run<8, 1>();
  if (vecs <= 16) return f.template run<16, 1>();
  if (vecs <= 32) return f.template run<32, 1>();
  if (vecs <= 64) return f.template run<64, 1>();
  constexpr int NV = kRegElements / kVec<TZ>;
  if (vecs <= 64 * NV) return f.template run<64, NV>();
  if (vecs <= 128 * NV) return f.template run<128, NV>();
  if (vecs <= 256 * NV) return f.template run<256, NV>();
  if (vecs <= 512 * NV) return f.template run<512, NV>();
  return f.template run<1024, NV>();
}

template <typename TS, typename TZ>
struct RowsForward {
  const Args& a;
  hipStream_t stream;
  template <int LPR, int NV>
  hipError_t run() const {
    typedef NormShape<TZ, LPR, NV> S;
    const int64_t steps = ceil_div(a.n, S::G);
    const int64_t per = ceil_div(steps, std::min(steps, kRegBlocks)) * S::G;
    hipLaunchKernelGGL((residual_norm_kernel<TS, TZ, LPR, NV>), dim3((unsigned)ceil_div(a.n, per)), dim3(S::BLOCK), 0,
                       stream, a, per, (uint32_t)std::min(a.gate_span, a.n));
    return hipGetLastError();
  }
};
template <typename TS, typename TZ>
struct RowsBackward {
  const Args& a;
  const Units& un;
  float* partial;
  float* gate;
  hipStream_t stream;
  template <int LPR, int NV>
  hipError_t run() const {
    typedef NormShape<TZ, LPR, NV> S;
    const dim3 grid((unsigned)std::min(un.units, kUnitBlocks));
    if (un.gate)
      hipLaunchKernelGGL((residual_norm_grad_kernel<TS, TZ, LPR, NV, true>), grid, dim3(S::BLOCK), 0, stream, a, un,
                         partial, gate);
    else
      hipLaunchKernelGGL((residual_norm_grad_kernel<TS, TZ, LPR, NV, false>), grid, dim3(S::BLOCK), 0, stream, a, un,
                         partial, gate);
    return hipGetLastError();
  }
};

template <typename TS, typename TZ>
static hipError_t forward_as(const Args& a, hipStream_t stream) {
  if (a.D <= kRegColumns) return with_shape<TZ>(a.D, RowsForward<TS, TZ>{a, stream});
  hipLaunchKernelGGL((residual_norm_wide_kernel<TS, TZ>), dim3((unsigned)std::min(a.n, kMaxRowGrid)), dim3(kRowBlock), 0,
                     stream, a);
  return hipGetLastError();
}

template <typename TS, typename TZ>
static hipError_t backward_as(const Args& a, void* ws, hipStream_t stream) {
  const NormRoom room = norm_room(a.n, a.D);
  float* partial = reinterpret_cast<float*>(static_cast<char*>(ws) + room.partial);
  float* gate = reinterpret_cast<float*>(static_cast<char*>(ws) + room.gate);
  float* means = reinterpret_cast<float*>(static_cast<char*>(ws) + room.means);
  const Units un = units_of(a);
  const bool params = a.dpost_weight || a.dpost_bias || a.dpre_weight || a.dpre_bias;
  const int64_t parts = std::min(un.units, kUnitBlocks);
  if (a.D <= kRegColumns) {
    const hipError_t e = with_shape<TZ>(a.D, RowsBackward<TS, TZ>{a, un, partial, gate, stream});
    if (e != hipSuccess) return e;
  } else {
    const unsigned rows = (unsigned)std::min(a.n, kMaxRowGrid);
    hipLaunchKernelGGL((residual_norm_means_kernel<TS, TZ>), dim3(rows), dim3(kRowBlock), 0, stream, a, means);
    // (the columns before the rows: dx may take dh's place, and dz dy's)
    if (params || un.gate) {
      const dim3 grid((unsigned)parts, (unsigned)ceil_div(a.D, kWave * kV));
      hipLaunchKernelGGL((residual_norm_columns_kernel<TS, TZ>), grid, dim3(kRowBlock), 0, stream, a,
                         (const float*)means, un, partial, gate);
    }
    if (a.dx || a.dz || (a.dgate && a.gate_span == 1))
      hipLaunchKernelGGL((residual_norm_rows_kernel<TS, TZ>), dim3(rows), dim3(kRowBlock), 0, stream, a,
                         (const float*)means);
  }
  const int64_t joined = un.gate && un.cuts > 1 ? un.units / un.cuts : 0;
  if ((params && !(parts == 1 && a.D <= kRegColumns)) || joined)
    hipLaunchKernelGGL(residual_norm_join_kernel, dim3((unsigned)ceil_div(a.D, kWave), (unsigned)(4 + joined)),
                       dim3(kJoinBlock), 0, stream, a, (const float*)partial, parts, un, (const float*)gate);
  return hipGetLastError();
}

// Calls f.run<stream's type, the others' type>().
template <typename F>
static hipError_t with_types(const Args& a, const F& f) {
  if (a.type == GBA_F32) return f.template run<float, float>();
  if (a.type == GBA_BF16) return a.stream_type == GBA_F32 ? f.template run<float, bf16_t>() : f.template run<bf16_t, bf16_t>();
  return a.stream_type == GBA_F32 ? f.template run<float, f16_t>() : f.template run<f16_t, f16_t>();
}
struct Forward {
  const Args& a;
  hipStream_t stream;
  template <typename TS, typename TZ>
  hipError_t run() const { return forward_as<TS, TZ>(a, stream); }
};
struct Backward {
  const Args& a;
  void* ws;
  hipStream_t stream;
  template <typename TS, typename TZ>
  hipError_t run() const { return backward_as<TS, TZ>(a, ws, stream); }
};

hipError_t launch_residual_norm(const Args& a, hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  return with_types(a, Forward{a, stream});
}

static __global__ void __launch_bounds__(kRowBlock) residual_norm_zero_kernel(Args a) {
  const float none[1] = {0.0f};
  const int64_t c = (int64_t)blockIdx.x * kRowBlock + threadIdx.x;
  if (c >= a.D) return;
  if (a.dpost_weight) store_part<1>(a.dpost_weight, a.grad_type, c, 1, none);
  if (a.dpost_bias) store_part<1>(a.dpost_bias, a.grad_type, c, 1, none);
  if (a.dpre_weight) store_part<1>(a.dpre_weight, a.grad_type, c, 1, none);
  if (a.dpre_bias) store_part<1>(a.dpre_bias, a.grad_type, c, 1, none);
}

hipError_t launch_residual_norm_grad(const Args& a, void* ws, hipStream_t stream) {
  if (a.n > 0) return with_types(a, Backward{a, ws, stream});
  hipLaunchKernelGGL(residual_norm_zero_kernel, dim3((unsigned)ceil_div(a.D, kRowBlock)), dim3(kRowBlock), 0, stream, a);
  return hipGetLastError();
}

}  // namespace gba
