// A block's output joined to the residual stream, and the stream normalised
// for the next block, row by row:
//   u = post(z),  h = alpha x + act(gate) u,  y = pre(h),
// post and pre each nothing, a layer norm or an RMS norm.
//
// Bound by bytes: 16,384 x 4096 bf16 106 us (537 MB, 5.1 TB/s, as a large copy); 8 rows
// of 2048 4.8 us of the GPU and 10 of the host.  A row is read once, held in registers
// over lanes or waves from its only read to its only write, and the next one is loaded
// meanwhile; rows wider than 8192 columns are read again for each sum (4000 x 16,384 bf16
// 220 us, 2.4 TB/s; before the rows were held, the first took 245).
#include "residual_norm.hpp"

namespace gba {

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

// ------------------------------------------------------ rows in registers
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
    row_total<LPR, WAVES>(t, s, buffer);
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
  row_total<LPR, WAVES>(t, s, buffer);
  rstd = 1.0f / sqrtf(t[0] / D + eps);
}

template <typename TS, typename TZ, int LPR, int NV>
__global__ void __launch_bounds__((NormShape<kVec<TZ>, LPR, NV>::BLOCK), 4)
residual_norm_kernel(Args a, int64_t per, uint32_t span) {
  typedef NormShape<kVec<TZ>, LPR, NV> S;
  constexpr int V = S::V;
  typedef typename VecOf<TS, V>::type stream_vec;
  typedef typename VecOf<TZ, V>::type vec;
  __shared__ float s_sum[2][1][S::WAVES];
  const int gl = threadIdx.x % LPR, grp = S::G == 1 ? 0 : threadIdx.x / LPR;   // (a row's addresses are then uniform)
  const RowPlace<V, LPR, NV, false> at(gl, a.D);
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
    if (each) load_gate_row(at, a.gate, a.gate_type, r * a.gate_stride, g);
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
      gate_factors(a.gate_kind, f);
    } else if (gated) {
      const int64_t g = (uint32_t)(active ? r : r1 - 1) / span;
      if (g != gate_row) {
        gate_row = g;
        load_gate_row(at, a.gate, a.gate_type, g * a.gate_stride, f);
        gate_factors(a.gate_kind, f);
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
    else if (LPR > kWave) __syncthreads();   // h may be x, and the last vectors overlap: all of the row has been read
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

// ------------------------------------------------------------- launching
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
    typedef NormShape<kVec<TZ>, LPR, NV> S;
    const int64_t steps = ceil_div(a.n, S::G);
    const int64_t per = ceil_div(steps, std::min(steps, kRegBlocks)) * S::G;
    hipLaunchKernelGGL((residual_norm_kernel<TS, TZ, LPR, NV>), dim3((unsigned)ceil_div(a.n, per)), dim3(S::BLOCK), 0,
                       stream, a, per, (uint32_t)std::min(a.gate_span, a.n));
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

struct Forward {
  const Args& a;
  hipStream_t stream;
  template <typename TS, typename TZ>
  hipError_t run() const { return forward_as<TS, TZ>(a, stream); }
};
hipError_t launch_residual_norm(const Args& a, hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  return with_types(a, Forward{a, stream});
}

}  // namespace gba
