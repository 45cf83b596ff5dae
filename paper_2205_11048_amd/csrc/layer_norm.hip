// Layer norm over the rows of a matrix and its gradient.
//
// A row stays in registers from its only read to its only write: 4 to 16
// elements per thread, the row spread over 1 to 64 lanes of a wave or 2 to 16
// waves, so that the mean, then the mean of the squared differences (forward)
// or the two sums (backward) are taken from registers.  Blocks stay on the
// chip and take rows in turn, so the weight and the bias are read once per
// block, and the weight's gradient is added up in registers over all the
// block's rows: one partial row per block goes to memory and a second launch
// adds the blocks' rows up in order.  Bound by the bytes of the rows: forward
// 20,011 x 1001 f32 26 us, 6.2 TB/s; backward 16,384 x 4096 bf16 72 us, 5.6, and
// 256,000 x 64 f32 31, 6.4, each with 4.6 for the join.  (A large copy reaches
// 4.9, a large fill 6.9.)  8 rows of 2048, one row's chain of latencies, take 4.1
// forward.
#include <algorithm>

#include "elements.hpp"
#include "gba_device.hpp"
#include "gba_internal.hpp"

namespace gba {

constexpr int kNormRowBlock = 256;           // rows read from memory again
constexpr int kNormRowWaves = kNormRowBlock / kWave;
constexpr int64_t kGradRowsPerBlock = 256;   // ... of a partial sum of the weight's gradient
constexpr int64_t kMaxRowGrid = 1 << 20;

constexpr int kPerThread = 16;               // elements of its rows a thread holds, forward
constexpr int kGradVecs = 2;                 // most 16-byte vectors of a row a thread holds, backward
constexpr int kRegBlock = 512;
constexpr int kWidest = 1024;                // most threads of a row
constexpr int64_t kRegGradBlocks = 512;      // most blocks of a gradient: two per compute unit
// Of so few steps of a block with several rows, one block takes all and writes the weight's gradient itself: 8 rows
// of 2048 bf16 8.9 us and 11.7 with a launch that joins blocks, 16 rows (four steps) 10.4 and 11.7, 32 (eight) 16.2 and
// 11.8; blocks of one row: 4 of 8000 14.9 and 12.1.
constexpr int64_t kOneBlockSteps = 4;
constexpr int64_t kRegBlocks = 2048;         // ... of a forward call

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

// ------------------------------------------------------ rows in registers
// Adds x over each aligned group of W lanes (W a power of two); every lane
// gets the sum.  Up to 16 lanes the exchange is a DPP operand of the addition.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  const int y = __builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true);
  return x + __int_as_float(y);
}
template <int W>
__device__ __forceinline__ float lanes_sum(float x) {
  if constexpr (W >= 2) x = dpp_add<0xB1>(x);    // lane ^ 1
  if constexpr (W >= 4) x = dpp_add<0x4E>(x);    // lane ^ 2
  if constexpr (W >= 8) x = dpp_add<0x141>(x);   // the other four of eight (all four hold one value)
  if constexpr (W >= 16) x = dpp_add<0x140>(x);  // the other eight of sixteen
  if constexpr (W >= 32) x += __shfl_xor(x, 16, kWave);
  if constexpr (W >= 64) x += __shfl_xor(x, 32, kWave);
  return x;
}

// How a row lies over the threads: LPR threads with NV vectors of V elements
// each, vector k of thread t at column (k * LPR + t) * V.  The last vector may
// pass the row's end: it is moved back to end there, its first `shift`
// elements belong to other threads and count for nothing (all V of them in a
// thread past the end); what is stored of them is what their owner stores.
// RU rows per thread group at a time.
template <typename T, int LPR, int NV>
struct RowShape {
  static constexpr int V = kVec<T>;
  static constexpr int E = V * NV;
  static constexpr int BLOCK = LPR > kRegBlock ? LPR : kRegBlock;
  static constexpr int G = BLOCK / LPR;         // thread groups of a block
  static constexpr int WAVES = BLOCK / kWave;
  static constexpr int RU = kPerThread / E;             // forward
  static constexpr int RU_GRAD = NV == 1 ? 2 : 1;       // backward
};

template <typename T, int LPR, int NV>
struct RowPlace {
  static constexpr int V = kVec<T>;
  int col[NV];     // first column of each vector
  int shift;       // foreign elements of the last one
  bool last;       // the last one holds elements of this thread
  bool tiny;       // rows narrower than a vector (LPR = NV = 1): element by element
  int D;
  __device__ __forceinline__ RowPlace(int gl, int width) : D(width) {
    tiny = width < V;
#pragma unroll
    for (int k = 0; k < NV; ++k) col[k] = (k * LPR + gl) * V;
    const int c = col[NV - 1];
    last = c < width;
    const int moved = tiny ? 0 : (c + V > width ? width - V : c);
    shift = c - moved < V ? c - moved : V;
    col[NV - 1] = moved;
  }
  __device__ __forceinline__ bool own(int k, int e) const {
    return k + 1 < NV || (tiny ? e < D : e >= shift);
  }
  template <typename P>
  __device__ __forceinline__ void load(const P* __restrict__ p, int k, float (&o)[V]) const {
    if (tiny) load_part<P, V>(p, D, o);
    else load_vec<P, V>(p + col[k], o);
  }
  // as it is in memory
  __device__ __forceinline__ typename VecOf<T, V>::type load_raw(const T* __restrict__ p, int k) const {
    typename VecOf<T, V>::type v;
    if (tiny) {
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = e < D ? p[e] : (T)0.0f;
    } else {
      v = *reinterpret_cast<const typename VecOf<T, V>::type*>(p + col[k]);
    }
    return v;
  }
  __device__ __forceinline__ void load(const void* __restrict__ p, int type, int k, float (&o)[V]) const {
    if (type == GBA_F32) load(static_cast<const float*>(p), k, o);
    else if (type == GBA_BF16) load(static_cast<const bf16_t*>(p), k, o);
    else load(static_cast<const f16_t*>(p), k, o);
  }
  // (past the caches: 20,011 x 1001 f32 forward 27 us, 32 through them.  With what
  // reads the output next, past the caches and through them: a second layer norm,
  // 2048 x 1024 bf16 12.5 and 12.5, 8192 x 1024 14.2 and 15.9, 8192 x 4096 49.7 and 44.9,
  // 16,384 x 4096 91 and 91; an addition, 8192 x 1024 17.4 and 18.6, 8192 x 4096 51.3 and
  // 50.6, 16,384 x 4096 104 and 116)
  __device__ __forceinline__ void store(T* __restrict__ p, int k, const float (&o)[V]) const {
    if (tiny) store_part<T, V>(p, D, o);
    else if (k + 1 < NV || last) store_vec<T, V, true>(p + col[k], o);
  }
};

// Adds each of x[0..N) over the LPR threads of a row.  Rows of several waves
// go through LDS, two buffers in turn so that one barrier a sum is enough.
template <int LPR, int WAVES, int N>
__device__ __forceinline__ void row_sum(float (&x)[N], float (*s)[N][WAVES], int& buffer) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = lanes_sum<(LPR < kWave ? LPR : kWave)>(x[i]);
  if constexpr (LPR > kWave) {
    constexpr int PER = LPR / kWave;
    const int w = threadIdx.x / kWave, w0 = w / PER * PER;
    if (lane_id() == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) s[buffer][i][w] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t = 0.0f;
#pragma unroll
      for (int k = 0; k < PER; ++k) t += s[buffer][i][w0 + k];
      x[i] = t;
    }
    buffer ^= 1;
  }
}

template <typename T, int LPR, int NV>
__global__ void __launch_bounds__((RowShape<T, LPR, NV>::BLOCK))
layer_norm_kernel(LayerNormArgs a) {
  typedef RowShape<T, LPR, NV> S;
  constexpr int V = S::V, RU = S::RU, ROWS = S::G * RU;
  __shared__ float s_sum[2][RU][S::WAVES];
  const int gl = threadIdx.x % LPR, grp = threadIdx.x / LPR;
  const RowPlace<T, LPR, NV> at(gl, a.D);
  float w[NV][V], b[NV][V];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      w[k][e] = 1.0f;
      b[k][e] = 0.0f;
    }
    if (a.weight) at.load(a.weight, a.weight_type, k, w[k]);
    if (a.bias) at.load(a.bias, a.weight_type, k, b[k]);
  }
  const float D = (float)a.D;
  int buffer = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.n; r0 += (int64_t)gridDim.x * ROWS) {
    float x[RU][NV][V], sum[RU];
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      const int64_t r = r0 + u * S::G + grp;
      const T* p = static_cast<const T*>(a.x) + (r < a.n ? r : a.n - 1) * a.x_stride;
#pragma unroll
      for (int k = 0; k < NV; ++k) at.load(p, k, x[u][k]);
    }
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      sum[u] = 0.0f;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) sum[u] += at.own(k, e) ? x[u][k][e] : 0.0f;
    }
    row_sum<LPR, S::WAVES>(sum, s_sum, buffer);
    float mean[RU];
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      mean[u] = sum[u] / D;
      sum[u] = 0.0f;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = at.own(k, e) ? x[u][k][e] - mean[u] : 0.0f;
          sum[u] = __builtin_fmaf(d, d, sum[u]);
        }
    }
    row_sum<LPR, S::WAVES>(sum, s_sum, buffer);
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      const int64_t r = r0 + u * S::G + grp;
      if (r >= a.n) continue;
      const float rstd = 1.0f / sqrtf(sum[u] / D + a.eps);
      if (gl == 0) {
        if (a.mean) a.mean[r] = mean[u];
        if (a.rstd) a.rstd[r] = rstd;
      }
      T* q = static_cast<T*>(a.y) + r * a.y_stride;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = __builtin_fmaf((x[u][k][e] - mean[u]) * rstd, w[k][e], b[k][e]);
        at.store(q, k, y);
      }
    }
  }
}

// The rows are kept as they are in memory and widened twice, and the next rows
// are asked for before the present ones are worked on.
template <typename T, int LPR, int NV>
__global__ void __launch_bounds__((RowShape<T, LPR, NV>::BLOCK), 4)
layer_norm_grad_kernel(LayerNormGradArgs a, float* __restrict__ partial) {
  typedef RowShape<T, LPR, NV> S;
  typedef typename VecOf<T, S::V>::type vec;
  constexpr int V = S::V, RU = S::RU_GRAD, ROWS = S::G * RU;
  // the block's sums of the weight's gradient: one row per wave or per group of several waves
  constexpr int TEAM = LPR < kWave ? kWave : LPR;
  constexpr int TEAMS = S::BLOCK / TEAM;
  constexpr int COLS = LPR * S::E;
  __shared__ float s_sum[2][2 * RU][S::WAVES];
  __shared__ float s_part[TEAMS > 1 ? TEAMS * COLS : 1];
  const int gl = threadIdx.x % LPR, grp = threadIdx.x / LPR;
  const RowPlace<T, LPR, NV> at(gl, a.D);
  float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      w[k][e] = 1.0f;
      dw[k][e] = db[k][e] = 0.0f;
    }
    if (a.weight) at.load(a.weight, a.weight_type, k, w[k]);
  }
  const float D = (float)a.D;
  int buffer = 0;
  vec x[RU][NV], g[RU][NV], xn[RU][NV], gn[RU][NV];
  float mean[RU], rstd[RU], mn[RU], rn[RU];
  auto load_rows = [&](int64_t r0, vec (&xv)[RU][NV], vec (&gv)[RU][NV], float (&m)[RU], float (&s)[RU]) {
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      const int64_t r = r0 + u * S::G + grp, rc = r < a.n ? r : a.n - 1;
      const T* p = static_cast<const T*>(a.x) + rc * a.x_stride;
      const T* q = static_cast<const T*>(a.dy) + rc * a.dy_stride;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        xv[u][k] = at.load_raw(p, k);
        gv[u][k] = at.load_raw(q, k);
      }
      m[u] = a.mean[rc];
      s[u] = a.rstd[rc];
    }
  };
  const int64_t step = (int64_t)gridDim.x * ROWS;
  int64_t r0 = (int64_t)blockIdx.x * ROWS;
  load_rows(r0, x, g, mean, rstd);
  for (; r0 < a.n; r0 += step) {
    const bool more = r0 + step < a.n;
    if (more) load_rows(r0 + step, xn, gn, mn, rn);
    float sum[2 * RU];
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      sum[2 * u] = sum[2 * u + 1] = 0.0f;
      if (r0 + u * S::G + grp >= a.n) continue;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float xh = ((float)x[u][k][e] - mean[u]) * rstd[u];
          // a foreign element adds 0 (what it adds to dw is not kept)
          const float gy = at.own(k, e) ? (float)g[u][k][e] : 0.0f;
          const float h = gy * w[k][e];
          sum[2 * u] += h;
          sum[2 * u + 1] = __builtin_fmaf(h, xh, sum[2 * u + 1]);
          dw[k][e] = __builtin_fmaf(gy, xh, dw[k][e]);
          db[k][e] += gy;
        }
    }
    if (a.dx) {
      row_sum<LPR, S::WAVES>(sum, s_sum, buffer);
#pragma unroll
      for (int u = 0; u < RU; ++u) {
        const int64_t r = r0 + u * S::G + grp;
        if (r >= a.n) continue;
        const float s1 = sum[2 * u] / D, s2 = sum[2 * u + 1] / D;
        T* q = static_cast<T*>(a.dx) + r * a.dx_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          float d[V];
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float xh = ((float)x[u][k][e] - mean[u]) * rstd[u];
            d[e] = rstd[u] * ((float)g[u][k][e] * w[k][e] - s1 - xh * s2);
          }
          at.store(q, k, d);
        }
      }
    }
    if (more) {
#pragma unroll
      for (int u = 0; u < RU; ++u) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          x[u][k] = xn[u][k];
          g[u][k] = gn[u][k];
        }
        mean[u] = mn[u];
        rstd[u] = rn[u];
      }
    }
  }
  if (!a.dweight && !a.dbias) return;
  float* out = partial + (int64_t)blockIdx.x * 2 * a.D;
  // the only block writes the sums themselves
  const bool only = gridDim.x == 1;
  auto write = [&](int which, int c, float t) {
    const float v[1] = {t};
    if (void* to = which ? a.dbias : a.dweight) store_part<1>(to, a.grad_type, c, 1, v);
  };
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float(&acc)[NV][V] = which ? db : dw;
    if constexpr (LPR < kWave) {
#pragma unroll
      for (int off = LPR; off < kWave; off <<= 1)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[0][e] += __shfl_xor(acc[0][e], off, kWave);   // (NV is 1)
    }
    if constexpr (TEAMS > 1) {
      if (which) __syncthreads();   // the first sums have been read
      if ((int)(threadIdx.x % TEAM) < LPR) {
        float* s = s_part + threadIdx.x / TEAM * COLS;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (at.own(k, e)) s[at.col[k] + e] = acc[k][e];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < a.D; c += S::BLOCK) {
        float t = 0.0f;
#pragma unroll
        for (int m = 0; m < TEAMS; ++m) t += s_part[m * COLS + c];
        if (only) write(which, c, t);
        else out[which * a.D + c] = t;
      }
    } else {
      if (only) {   // (a single row)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (at.own(k, e)) write(which, at.col[k] + e, acc[k][e]);
      } else {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (at.own(k, e)) out[which * a.D + at.col[k] + e] = acc[k][e];
      }
    }
  }
}

// -------------------------------------------- rows read from memory again
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

// Rows of any width, a block per row, read again for every pass over it: three
// reads and a write forward (4096 x 20,000 bf16 100 us, 656 MB at 6.6 TB/s; f32 219,
// 1311 MB at 6.0, where 16,384 columns in registers move 2148 MB once in 379).
// Backward (4096 x 10,000) the columns' partial sums take 59 us in bf16 and f32
// alike (164 and 328 MB: a wave's 64 rows one after another), the rows 58 and 124
// (410 and 819 MB at 7.0 and 6.6 TB/s), the join 4.8.
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

// dweight and dbias from the partial sums of `parts` blocks of rows: 64
// columns a block, each wave a share of the parts.
constexpr int kJoinBlock = 1024;
constexpr int kJoinWaves = kJoinBlock / kWave;
__global__ void __launch_bounds__(kJoinBlock)
layer_norm_join_kernel(const float* __restrict__ partial, int64_t parts, int32_t D, void* dweight, void* dbias,
                       int32_t type) {
  __shared__ float s_sum[kJoinWaves][kWave];
  const int w = threadIdx.x / kWave, lane = lane_id();
  const int64_t i = (int64_t)blockIdx.x * kWave + lane;
  const int64_t width = 2 * (int64_t)D;
  float s[1] = {0.0f};
  if (i < width) {
#pragma unroll 8
    for (int64_t p = w; p < parts; p += kJoinWaves) s[0] += partial[p * width + i];
  }
  s_sum[w][lane] = s[0];
  __syncthreads();
  if (w != 0 || i >= width) return;
  s[0] = 0.0f;
#pragma unroll
  for (int k = 0; k < kJoinWaves; ++k) s[0] += s_sum[k][lane];
  void* out = i < D ? dweight : dbias;
  if (out) store_part<1>(out, type, i < D ? i : i - D, 1, s);
}

// ------------------------------------------------------------- launching
// Widest rows held in registers.
constexpr int kForwardColumns = kWidest * kPerThread;
constexpr int kGradColumns = kWidest * kGradVecs * kVec<float>;

// Partial rows of a gradient: at most one per row and per resident block of
// rows in registers, else one per kGradRowsPerBlock rows.
size_t layer_norm_grad_workspace_bytes(int64_t n, int32_t D) {
  const int64_t parts = D <= kGradColumns ? std::min(n, kRegGradBlocks) : ceil_div(n, kGradRowsPerBlock);
  return align_up((size_t)parts * 2 * (size_t)D * sizeof(float)) + 256;
}

template <typename T, int LPR, int NV>
static hipError_t forward_in(const LayerNormArgs& a, hipStream_t stream) {
  typedef RowShape<T, LPR, NV> S;
  const int64_t blocks = std::min(ceil_div(a.n, S::G * S::RU), kRegBlocks);
  hipLaunchKernelGGL((layer_norm_kernel<T, LPR, NV>), dim3((unsigned)blocks), dim3(S::BLOCK), 0, stream, a);
  return hipGetLastError();
}
template <typename T, int LPR, int NV>
static hipError_t backward_in(const LayerNormGradArgs& a, float* partial, int64_t* parts, hipStream_t stream) {
  typedef RowShape<T, LPR, NV> S;
  const int64_t steps = ceil_div(a.n, S::G * S::RU_GRAD);
  const int64_t blocks = S::G > 1 && steps <= kOneBlockSteps ? 1 : std::min(steps, kRegGradBlocks);
  *parts = blocks;
  hipLaunchKernelGGL((layer_norm_grad_kernel<T, LPR, NV>), dim3((unsigned)blocks), dim3(S::BLOCK), 0, stream, a,
                     partial);
  return hipGetLastError();
}

// Calls f.run<LPR, NV>() for the shape of rows of `vecs` vectors: as few
// threads as hold the row, one vector each up to a wave (more rows per wave
// and more of them in flight then), up to M each beyond; MOST vectors at most.
template <int M, int MOST, typename F>
static hipError_t with_shape(int vecs, const F& f) {
  if (vecs <= 1) return f.template run<1, 1>();
  if (vecs <= 2) return f.template run<2, 1>();
  if (vecs <= 4) return f.template run<4, 1>();
  if (vecs <= 8) return f.template run<8, 1>();
  if (vecs <= 16) return f.template run<16, 1>();
  if (vecs <= 32) return f.template run<32, 1>();
  if (vecs <= 64) return f.template run<64, 1>();
  if (vecs <= 128) return f.template run<64, 2>();
  if constexpr (M == 4) {
    if (vecs <= 192) return f.template run<64, 3>();
    if (vecs <= 256) return f.template run<64, 4>();
    if (vecs <= 384) return f.template run<128, 3>();
    if (vecs <= 512) return f.template run<128, 4>();
    if (vecs <= 768) return f.template run<256, 3>();
    if (vecs <= 1024) return f.template run<256, 4>();
    if (vecs <= 1536) return f.template run<512, 3>();
    if (vecs <= 2048) return f.template run<512, 4>();
    if (vecs <= 3 * 1024) return f.template run<1024, 3>();
    return f.template run<1024, 4>();
  } else {
    static_assert(M == 2, "two vectors a thread, or four");
    if (vecs <= 256) return f.template run<128, 2>();
    if (vecs <= 512) return f.template run<256, 2>();
    if constexpr (MOST <= 1024) {
      return f.template run<512, 2>();
    } else {
      if (vecs <= 1024) return f.template run<512, 2>();
      return f.template run<1024, 2>();
    }
  }
}

template <typename T>
struct ForwardCall {
  const LayerNormArgs& a;
  hipStream_t stream;
  template <int LPR, int NV>
  hipError_t run() const { return forward_in<T, LPR, NV>(a, stream); }
};
template <typename T>
struct BackwardCall {
  const LayerNormGradArgs& a;
  float* partial;
  int64_t* parts;
  hipStream_t stream;
  template <int LPR, int NV>
  hipError_t run() const { return backward_in<T, LPR, NV>(a, partial, parts, stream); }
};

template <typename T>
static hipError_t forward_as(const LayerNormArgs& a, hipStream_t stream) {
  if (a.D <= kForwardColumns)
    return with_shape<kPerThread / kVec<T>, kForwardColumns / kVec<T>>((int)ceil_div(a.D, kVec<T>), ForwardCall<T>{a, stream});
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
static hipError_t backward_as(const LayerNormGradArgs& a, float* partial, int64_t* parts, hipStream_t stream) {
  if (a.D <= kGradColumns)
    return with_shape<kGradVecs, kGradColumns / kVec<T>>((int)ceil_div(a.D, kVec<T>), BackwardCall<T>{a, partial, parts, stream});
  *parts = ceil_div(a.n, kGradRowsPerBlock);
  // the columns first: dx may take dy's place
  if (a.dweight || a.dbias) {
    const unsigned slices = (unsigned)ceil_div(a.D, kWave * kVec<T>);
    hipLaunchKernelGGL(layer_norm_columns_kernel<T>, dim3((unsigned)*parts, slices), dim3(kNormRowBlock), 0, stream, a,
                       partial);
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
  int64_t parts = 0;
  if (a.n > 0 && (a.dx || a.dweight || a.dbias)) {
    const hipError_t e = a.type == GBA_F32    ? backward_as<float>(a, partial, &parts, stream)
                         : a.type == GBA_BF16 ? backward_as<bf16_t>(a, partial, &parts, stream)
                                              : backward_as<f16_t>(a, partial, &parts, stream);
    if (e != hipSuccess) return e;
  }
  if ((!a.dweight && !a.dbias) || (parts == 1 && a.D <= kGradColumns)) return hipSuccess;
  hipLaunchKernelGGL(layer_norm_join_kernel, dim3((unsigned)ceil_div(2 * (int64_t)a.D, kWave)), dim3(kJoinBlock), 0,
                     stream, (const float*)partial, parts, a.D, a.dweight, a.dbias, a.grad_type);
  return hipGetLastError();
}

}  // namespace gba
