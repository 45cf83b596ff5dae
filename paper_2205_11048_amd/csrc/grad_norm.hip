// The global norm of many gradient tensors and clipping by it: the squares of
// every element are summed in float64 (no finite float overflows it, and the
// order matters at the 1e-16 level only), chunk by chunk in a fixed order, and
// every tensor is scaled by min(1, max_norm / norm) on its way out.
//
// The list of tensors is cut into chunks of kChunkBytes on the host, once:
// a chunk's record holds all a block needs, so a block's first load already
// leads to its data and tensors of any sizes give even work.
//
// Bound by bytes, of which the second pass reads again what the 256 MB cache no
// longer holds: 200 M f32 elements 120 us for the sum (6.6 TB/s) and 285 for the
// scaling (5.6 TB/s); small lists by the two launches (65,536 elements 3.0 and
// 5.0 us).
#include <algorithm>
#include <cmath>
#include <limits>

#include "elements.hpp"
#include "gba_device.hpp"
#include "gba_internal.hpp"

namespace gba {

constexpr int kNormBlock = 256;
constexpr int kNormWaves = kNormBlock / kWave;
constexpr int kChunkBytes = 1 << 15;   // of a chunk, as it is read
constexpr int64_t kNormMaxBlocks = 512;   // two a compute unit: 421 us at 200 M f32 elements, 1024 447, 2048 489

// One chunk of one tensor, in the device list.
struct TensorChunk {
  const void* grad;      // the chunk's first element
  void* out;             // ... and where it goes (null: nowhere)
  const int64_t* rows;   // device word: rows of the tensor that count (null: all)
  int64_t at;            // the chunk's first element in its tensor
  int64_t width;         // elements of a row
  int32_t count;         // elements of the chunk
  int32_t types;         // grad_type | out_type << 8 | in place << 16
};
static_assert(sizeof(TensorChunk) == 48, "the list's record");

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

static int64_t norm_blocks(int64_t chunks) { return std::min(chunks, kNormMaxBlocks); }

static int size_of(int type) { return type == GBA_F32 ? 4 : 2; }

int64_t tensor_chunks(const gba_tensor* t, int32_t T) {
  int64_t c = 0;
  for (int32_t i = 0; i < T; ++i) c += ceil_div(t[i].n * size_of(t[i].grad_type), kChunkBytes);
  return c;
}
size_t tensor_list_bytes(int64_t chunks) { return (size_t)chunks * sizeof(TensorChunk); }
size_t grad_norm_workspace_bytes(int64_t chunks) { return (size_t)(norm_blocks(chunks) + 1) * sizeof(double); }

void fill_tensor_list(const gba_tensor* t, int32_t T, void* list) {
  TensorChunk* c = static_cast<TensorChunk*>(list);
  for (int32_t i = 0; i < T; ++i) {
    const int64_t most = kChunkBytes / size_of(t[i].grad_type);
    for (int64_t at = 0; at < t[i].n; at += most, ++c) {
      c->grad = static_cast<const char*>(t[i].grad) + at * size_of(t[i].grad_type);
      c->out = t[i].out ? static_cast<char*>(t[i].out) + at * size_of(t[i].out_type) : nullptr;
      c->rows = t[i].rows;
      c->at = at;
      c->width = t[i].rows ? t[i].width : 1;
      c->count = (int32_t)std::min(most, t[i].n - at);
      const bool in_place = t[i].out == t[i].grad;
      c->types = t[i].grad_type | t[i].out_type << 8 | (in_place ? 1 : 0) << 16;
    }
  }
}

// Elements of the chunk that count.
__device__ __forceinline__ int chunk_count(const TensorChunk& c) {
  if (!c.rows) return c.count;
  const int64_t rows = *c.rows;
  if (rows <= 0) return 0;
  // rows * width may not fit 64 bits: compare before multiplying
  const int64_t need = (c.at + c.count + c.width - 1) / c.width;
  if (rows >= need) return c.count;
  const int64_t end = rows * c.width - c.at;
  return end <= 0 ? 0 : end < c.count ? (int)end : c.count;
}

// Sum over the block, in a fixed order; every thread gets it.
__device__ __forceinline__ double block_sum(double x, double* s_wave) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) x += __shfl_xor(x, off, kWave);
  if (lane_id() == 0) s_wave[threadIdx.x / kWave] = x;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kNormWaves; ++w) s += s_wave[w];
  return s;
}

// A chunk as a block holds it, in vectors of V elements: vector k * kNormBlock
// + t with thread t, all asked for at once; what is left of a chunk that is
// not whole vectors is one element a thread.
template <typename T, int V>
struct ChunkData {
  static constexpr int N = kChunkBytes / (int)sizeof(T) / V / kNormBlock;   // vectors of a thread
  typename VecOf<T, V>::type x[N];
  T rest;

  __device__ __forceinline__ void load(const void* grad, int count) {
    const T* g = static_cast<const T*>(grad);
    const int whole = count / V;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int u = k * kNormBlock + threadIdx.x;
      x[k] = u < whole ? *reinterpret_cast<const typename VecOf<T, V>::type*>(g + u * V) : typename VecOf<T, V>::type{};
    }
    const int left = whole * V + threadIdx.x;
    rest = left < count ? g[left] : (T)0.0f;
  }
  __device__ __forceinline__ double squares() const {
    double s = (double)(float)rest * (double)(float)rest;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const double v = (double)(float)x[k][e];
        s = __builtin_fma(v, v, s);
      }
    return s;
  }
  // (past the caches, which then keep what is still to be read: 200 M f32 elements 421 us, 432 through them)
  template <typename O>
  __device__ __forceinline__ void store(void* to, int count, float first, float second) const {
    O* out = static_cast<O*>(to);
    const int whole = count / V;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int u = k * kNormBlock + threadIdx.x;
      typename VecOf<O, V>::type y;
#pragma unroll
      for (int e = 0; e < V; ++e) y[e] = (O)((float)x[k][e] * first * second);
      typename VecOf<O, V>::type* p = reinterpret_cast<typename VecOf<O, V>::type*>(out + u * V);
      if (u < whole) __builtin_nontemporal_store(y, p);
    }
    const int left = whole * V + threadIdx.x;
    if (left < count) out[left] = (O)((float)rest * first * second);
  }
};

template <typename T>
__device__ __forceinline__ double chunk_squares(const TensorChunk& c, int count) {
  ChunkData<T, kVec<T>> d;
  d.load(c.grad, count);
  return d.squares();
}

__global__ void __launch_bounds__(kNormBlock)
grad_squares_kernel(const TensorChunk* __restrict__ list, int64_t chunks, double* __restrict__ partial) {
  __shared__ double s_wave[kNormWaves];
  double s = 0.0;
  for (int64_t i = blockIdx.x; i < chunks; i += gridDim.x) {
    const TensorChunk c = list[i];
    const int count = chunk_count(c), type = c.types & 255;
    if (type == GBA_F32) s += chunk_squares<float>(c, count);
    else if (type == GBA_BF16) s += chunk_squares<bf16_t>(c, count);
    else s += chunk_squares<f16_t>(c, count);
  }
  s = block_sum(s, s_wave);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// The whole sum from the blocks' partial sums (every block of a launch gets
// the same bits).
__device__ __forceinline__ double total_squares(const double* __restrict__ partial, int blocks, double* s_wave) {
  double s = 0.0;
  for (int i = threadIdx.x; i < blocks; i += kNormBlock) s += partial[i];
  return block_sum(s, s_wave);
}

__global__ void __launch_bounds__(kNormBlock)
grad_norm_kernel(const double* __restrict__ partial, int blocks, float* __restrict__ norm, int32_t* err) {
  __shared__ double s_wave[kNormWaves];
  const double n = sqrt(total_squares(partial, blocks, s_wave));
  if (threadIdx.x == 0) {
    *norm = (float)n;
    if (!isfinite(n)) raise_error(err, GBA_DERR_NONFINITE);
  }
}

// What the coefficient is waited for: the first chunk of a block is on its way
// when the block adds up the partial sums.  The elements are multiplied by
// `first`, rounded to 24 bits, and then by `second`, a power of two: 1, or
// 2^-126 where the coefficient is below float's normal range and would have
// fewer bits there (elements of 1e38 whose norm is 1e40 are still gradients).
struct Coefficient {
  const double* partial;
  int blocks;
  double max_norm;
  float* norm;
  float* coef_out;
  int32_t* err;
  double* s_wave;
  float value, first, second;
  bool known, finite;
  __device__ __forceinline__ void get() {
    if (known) return;
    known = true;
    const double n = sqrt(total_squares(partial, blocks, s_wave));
    finite = isfinite(n);
    const double c = !finite ? 0.0 : n > max_norm ? max_norm / n : 1.0;
    const bool small = c < 0x1p-126;
    value = (float)c;
    first = small ? (float)(c * 0x1p126) : value;
    second = small ? 0x1p-126f : 1.0f;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      *norm = (float)n;
      if (coef_out) *coef_out = value;
      if (!finite) raise_error(err, GBA_DERR_NONFINITE);
    }
  }
};

// The vectors have 16 bytes in the wider of the two types, so that both the
// loads and the stores of a wave are without gaps.
template <typename T, typename O>
__device__ __forceinline__ void clip_chunk(const TensorChunk& c, int count, Coefficient& f) {
  constexpr int V = kVec<T> < kVec<O> ? kVec<T> : kVec<O>;
  ChunkData<T, V> d;
  d.load(c.grad, count);
  f.get();
  if (f.finite && !(f.value == 1.0f && c.types >> 16))   // (in place with nothing to scale)
    d.template store<O>(c.out, count, f.first, f.second);
}
template <typename T>
__device__ __forceinline__ void clip_chunk(const TensorChunk& c, int count, Coefficient& f) {
  const int type = c.types >> 8 & 255;
  if (type == GBA_F32) clip_chunk<T, float>(c, count, f);
  else if (type == GBA_BF16) clip_chunk<T, bf16_t>(c, count, f);
  else clip_chunk<T, f16_t>(c, count, f);
}

// A block takes the chunks that the same block of the sum took (their bytes
// are in the caches of its part of the chip, if anywhere), the last first.
__global__ void __launch_bounds__(kNormBlock)
clip_kernel(const TensorChunk* __restrict__ list, int64_t chunks, const double* __restrict__ partial, int blocks,
            double max_norm, float* __restrict__ norm, float* __restrict__ coef_out, int32_t* err) {
  __shared__ double s_wave[kNormWaves];
  Coefficient f{partial, blocks, max_norm, norm, coef_out, err, s_wave, 1.0f, 1.0f, 1.0f, false, true};
  const int64_t rounds = (chunks + gridDim.x - 1) / gridDim.x;
  for (int64_t r = rounds - 1; r >= 0; --r) {
    const int64_t i = r * gridDim.x + blockIdx.x;
    if (i >= chunks) continue;
    const TensorChunk c = list[i];
    if (!c.out || (f.known && f.value == 1.0f && c.types >> 16)) continue;
    const int count = chunk_count(c), type = c.types & 255;
    if (type == GBA_F32) clip_chunk<float>(c, count, f);
    else if (type == GBA_BF16) clip_chunk<bf16_t>(c, count, f);
    else clip_chunk<f16_t>(c, count, f);
    if (!f.finite) return;
  }
  f.get();
}

static hipError_t launch_squares(const void* list, int64_t chunks, double* partial, hipStream_t stream) {
  if (chunks == 0) return hipSuccess;
  hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)norm_blocks(chunks)), dim3(kNormBlock), 0, stream,
                     static_cast<const TensorChunk*>(list), chunks, partial);
  return hipGetLastError();
}

hipError_t launch_grad_norm(const void* list, int64_t chunks, float* norm, void* ws, int32_t* err, hipStream_t stream) {
  double* partial = static_cast<double*>(ws);
  const hipError_t e = launch_squares(list, chunks, partial, stream);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kNormBlock), 0, stream, (const double*)partial,
                     (int)norm_blocks(chunks), norm, err);
  return hipGetLastError();
}

hipError_t launch_clip_grads(const void* list, int64_t chunks, double max_norm, float* norm, float* coef, void* ws,
                             int32_t* err, hipStream_t stream) {
  double* partial = static_cast<double*>(ws);
  const hipError_t e = launch_squares(list, chunks, partial, stream);
  if (e != hipSuccess) return e;
  const int64_t blocks = norm_blocks(chunks);
  hipLaunchKernelGGL(clip_kernel, dim3((unsigned)std::max<int64_t>(blocks, 1)), dim3(kNormBlock), 0, stream,
                     static_cast<const TensorChunk*>(list), chunks, (const double*)partial, (int)blocks, max_norm, norm,
                     coef, err);
  return hipGetLastError();
}

}  // namespace gba
