// Layer norm over the rows of a matrix and its gradient.
#include <algorithm>

#include "elements.hpp"
#include "gba_device.hpp"
#include "gba_internal.hpp"

namespace gba {

constexpr int kNormRowBlock = 256;
constexpr int kNormRowWaves = kNormRowBlock / kWave;
constexpr int64_t kGradRowsPerBlock = 256;   // rows of a partial sum of the weight's gradient
constexpr int64_t kMaxRowGrid = 1 << 20;

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

// Sums of two values over the block; every thread gets them.
__device__ __forceinline__ void block_sum2(float& a, float& b, float (*s)[kNormRowWaves]) {
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
  for (int k = 0; k < kNormRowWaves; ++k) {
    a += s[0][k];
    b += s[1][k];
  }
}

// Rows of any width, a block per row, read again for every pass over it.
template <typename T>
__global__ void __launch_bounds__(kNormRowBlock)
layer_norm_wide_kernel(LayerNormArgs a) {
  constexpr int V = kVec<T>;
  __shared__ float s_sum[2][kNormRowWaves];
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
    float sum = 0.0f, unused = 0.0f;
    for (int c = threadIdx.x * V; c < a.D; c += kNormRowBlock * V) {
      float v[V];
      load_part<T, V>(x + c, a.D - c, v);
#pragma unroll
      for (int e = 0; e < V; ++e) sum += v[e];
    }
    block_sum2(sum, unused, s_sum);
    const float mean = sum / (float)a.D;
    float sq = 0.0f;
    for (int c = threadIdx.x * V; c < a.D; c += kNormRowBlock * V) {
      float v[V];
      load_part<T, V>(x + c, a.D - c, v);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = c + e < a.D ? v[e] - mean : 0.0f;
        sq = __builtin_fmaf(d, d, sq);
      }
    }
    block_sum2(sq, unused, s_sum);
    const float rstd = 1.0f / sqrtf(sq / (float)a.D + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    for (int c = threadIdx.x * V; c < a.D; c += kNormRowBlock * V) {
      const int count = a.D - c;
      float v[V], w[V], b[V];
      load_part<T, V>(x + c, count, v);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        w[e] = 1.0f;
        b[e] = 0.0f;
      }
      if (a.weight) load_part<V>(a.weight, a.weight_type, c, count, w);
      if (a.bias) load_part<V>(a.bias, a.weight_type, c, count, b);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = __builtin_fmaf((v[e] - mean) * rstd, w[e], b[e]);
      store_part<T, V>(y + c, count, v);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kNormRowBlock)
layer_norm_dx_wide_kernel(LayerNormGradArgs a) {
  constexpr int V = kVec<T>;
  __shared__ float s_sum[2][kNormRowWaves];
  const float inv = 1.0f / (float)a.D;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
    T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x * V; c < a.D; c += kNormRowBlock * V) {
      const int count = a.D - c;
      float v[V], g[V], w[V];
      load_part<T, V>(x + c, count, v);
      load_part<T, V>(dy + c, count, g);
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = 1.0f;
      if (a.weight) load_part<V>(a.weight, a.weight_type, c, count, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float h = g[e] * w[e];   // past the row's end g is 0
        s1 += h;
        s2 = __builtin_fmaf(h, (v[e] - mean) * rstd, s2);
      }
    }
    block_sum2(s1, s2, s_sum);
    s1 *= inv;
    s2 *= inv;
    for (int c = threadIdx.x * V; c < a.D; c += kNormRowBlock * V) {
      const int count = a.D - c;
      float v[V], g[V], w[V];
      load_part<T, V>(x + c, count, v);
      load_part<T, V>(dy + c, count, g);
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = 1.0f;
      if (a.weight) load_part<V>(a.weight, a.weight_type, c, count, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float xh = (v[e] - mean) * rstd;
        v[e] = rstd * (g[e] * w[e] - s1 - xh * s2);
      }
      store_part<T, V>(dx + c, count, v);
    }
  }
}

// Partial sums of the weight's and the bias's gradient: a wave per slice of
// 64 vectors of columns and a block's rows, four waves' sums joined in LDS.
template <typename T>
__global__ void __launch_bounds__(kNormRowBlock)
layer_norm_columns_kernel(LayerNormGradArgs a, float* __restrict__ partial) {
  constexpr int V = kVec<T>;
  __shared__ float s_part[kNormRowWaves][2][kWave * V];
  const int w = threadIdx.x / kWave, lane = lane_id();
  const int c = (int)blockIdx.y * (kWave * V) + lane * V;
  const int64_t r0 = (int64_t)blockIdx.x * kGradRowsPerBlock;
  const int64_t r1 = r0 + kGradRowsPerBlock < a.n ? r0 + kGradRowsPerBlock : a.n;
  float dw[V] = {}, db[V] = {};
  if (c < a.D) {
    for (int64_t row = r0 + w; row < r1; row += kNormRowWaves) {
      float v[V], g[V];
      load_part<T, V>(static_cast<const T*>(a.x) + row * a.x_stride + c, a.D - c, v);
      load_part<T, V>(static_cast<const T*>(a.dy) + row * a.dy_stride + c, a.D - c, g);
      const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        dw[e] = __builtin_fmaf(g[e], (v[e] - mean) * rstd, dw[e]);
        db[e] += g[e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) {
    s_part[w][0][lane * V + e] = dw[e];
    s_part[w][1][lane * V + e] = db[e];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * kWave * V; i += kNormRowBlock) {
    const int which = i / (kWave * V), col = i % (kWave * V);
    const int64_t cc = (int64_t)blockIdx.y * (kWave * V) + col;
    if (cc >= a.D) continue;
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < kNormRowWaves; ++k) s += s_part[k][which][col];
    partial[((int64_t)blockIdx.x * 2 + which) * a.D + cc] = s;
  }
}

// dweight and dbias from the partial sums of `parts` blocks of rows.
__global__ void __launch_bounds__(kNormRowBlock)
layer_norm_join_kernel(const float* __restrict__ partial, int64_t parts, int32_t D, void* dweight, void* dbias,
                       int32_t type) {
  const int64_t i = (int64_t)blockIdx.x * kNormRowBlock + threadIdx.x;
  if (i >= 2 * (int64_t)D) return;
  void* out = i < D ? dweight : dbias;
  if (!out) return;
  float s[1] = {0.0f};
  for (int64_t p = 0; p < parts; ++p) s[0] += partial[p * 2 * D + i];
  store_part<1>(out, type, i < D ? i : i - D, 1, s);
}

static int64_t grad_parts(int64_t n) { return ceil_div(n, kGradRowsPerBlock); }

size_t layer_norm_grad_workspace_bytes(int64_t n, int32_t D) {
  return align_up((size_t)grad_parts(n) * 2 * (size_t)D * sizeof(float)) + 256;
}

template <typename T>
static hipError_t forward_as(const LayerNormArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(layer_norm_wide_kernel<T>, dim3((unsigned)std::min(a.n, kMaxRowGrid)), dim3(kNormRowBlock), 0,
                     stream, a);
  return hipGetLastError();
}

hipError_t launch_layer_norm(const LayerNormArgs& a, hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  if (a.type == GBA_F32) return forward_as<float>(a, stream);
  if (a.type == GBA_BF16) return forward_as<bf16_t>(a, stream);
  return forward_as<f16_t>(a, stream);
}

template <typename T>
static hipError_t backward_as(const LayerNormGradArgs& a, float* partial, hipStream_t stream) {
  // the columns first: dx may take dy's place
  if (a.dweight || a.dbias) {
    const unsigned slices = (unsigned)ceil_div(a.D, kWave * kVec<T>);
    hipLaunchKernelGGL(layer_norm_columns_kernel<T>, dim3((unsigned)grad_parts(a.n), slices), dim3(kNormRowBlock), 0,
                       stream, a, partial);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.dx) return hipSuccess;
  hipLaunchKernelGGL(layer_norm_dx_wide_kernel<T>, dim3((unsigned)std::min(a.n, kMaxRowGrid)), dim3(kNormRowBlock),
                     0, stream, a);
  return hipGetLastError();
}

hipError_t launch_layer_norm_grad(const LayerNormGradArgs& a, void* ws, hipStream_t stream) {
  float* partial = static_cast<float*>(ws);
  hipError_t e = hipSuccess;
  if (a.n > 0) {
    e = a.type == GBA_F32    ? backward_as<float>(a, partial, stream)
        : a.type == GBA_BF16 ? backward_as<bf16_t>(a, partial, stream)
                             : backward_as<f16_t>(a, partial, stream);
    if (e != hipSuccess) return e;
  }
  if (!a.dweight && !a.dbias) return hipSuccess;
  hipLaunchKernelGGL(layer_norm_join_kernel, dim3((unsigned)ceil_div(2 * (int64_t)a.D, kNormRowBlock)),
                     dim3(kNormRowBlock), 0, stream, (const float*)partial, grad_parts(a.n), a.D, a.dweight, a.dbias,
                     a.grad_type);
  return hipGetLastError();
}

}  // namespace gba
