// The global norm of many gradient tensors and clipping by it: the squares of
// every element are summed in float64 (no finite float overflows it, and the
// order matters at the 1e-16 level only), chunk by chunk in a fixed order, and
// every tensor is scaled by min(1, max_norm / norm) on its way out.
//
// The list of tensors is cut into chunks of kChunk elements on the host, once:
// a chunk's record holds all a block needs, so a block's first load already
// leads to its data and tensors of any sizes give even work.
#include <algorithm>
#include <cmath>
#include <limits>

#include "elements.hpp"
#include "gba_device.hpp"
#include "gba_internal.hpp"

namespace gba {

constexpr int kNormBlock = 256;
constexpr int kNormWaves = kNormBlock / kWave;
constexpr int kChunk = 8192;           // elements of a chunk
constexpr int64_t kNormMaxBlocks = 2048;

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

int64_t tensor_chunks(const gba_tensor* t, int32_t T) {
  int64_t c = 0;
  for (int32_t i = 0; i < T; ++i) c += ceil_div(t[i].n, kChunk);
  return c;
}
size_t tensor_list_bytes(int64_t chunks) { return (size_t)chunks * sizeof(TensorChunk); }
size_t grad_norm_workspace_bytes(int64_t chunks) { return (size_t)(norm_blocks(chunks) + 1) * sizeof(double); }

void fill_tensor_list(const gba_tensor* t, int32_t T, void* list) {
  TensorChunk* c = static_cast<TensorChunk*>(list);
  auto size = [](int type) { return type == GBA_F32 ? 4 : 2; };
  for (int32_t i = 0; i < T; ++i) {
    for (int64_t at = 0; at < t[i].n; at += kChunk, ++c) {
      c->grad = static_cast<const char*>(t[i].grad) + at * size(t[i].grad_type);
      c->out = t[i].out ? static_cast<char*>(t[i].out) + at * size(t[i].out_type) : nullptr;
      c->rows = t[i].rows;
      c->at = at;
      c->width = t[i].rows ? t[i].width : 1;
      c->count = (int32_t)std::min<int64_t>(kChunk, t[i].n - at);
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

// A chunk as a block holds it: 16-byte units, unit k * kNormBlock + t with
// thread t, all asked for at once; what is left of a chunk that is not whole
// units (fewer than eight elements) is one element a thread.
typedef VecOf<uint16_t, 8>::type unit_t;
constexpr int kUnits = kChunk * 4 / 16 / kNormBlock;   // of a thread, of 4-byte elements
struct ChunkData {
  unit_t unit[kUnits];
  float rest;
};

template <typename T>
__device__ __forceinline__ void load_chunk(const TensorChunk& c, int count, ChunkData& d) {
  constexpr int V = kVec<T>;
  const T* g = static_cast<const T*>(c.grad);
  const int units = count / V;
#pragma unroll
  for (int k = 0; k < kChunk / V / kNormBlock; ++k) {
    const int u = k * kNormBlock + threadIdx.x;
    d.unit[k] = u < units ? *reinterpret_cast<const unit_t*>(g + u * V) : unit_t{};
  }
  const int left = units * V + threadIdx.x;
  d.rest = left < count ? (float)g[left] : 0.0f;
}
__device__ __forceinline__ void load_chunk(const TensorChunk& c, int count, ChunkData& d) {
  const int type = c.types & 255;
  if (type == GBA_F32) load_chunk<float>(c, count, d);
  else if (type == GBA_BF16) load_chunk<bf16_t>(c, count, d);
  else load_chunk<f16_t>(c, count, d);
}

template <typename T>
__device__ __forceinline__ void unpack(const unit_t& unit, float (&v)[kVec<T>]) {
  typedef typename VecOf<T, kVec<T>>::type vec;
  const vec x = __builtin_bit_cast(vec, unit);
#pragma unroll
  for (int e = 0; e < kVec<T>; ++e) v[e] = (float)x[e];
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const ChunkData& d) {
  double s = (double)d.rest * (double)d.rest;
#pragma unroll
  for (int k = 0; k < kChunk / kVec<T> / kNormBlock; ++k) {
    float v[kVec<T>];
    unpack<T>(d.unit[k], v);
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) s = __builtin_fma((double)v[e], (double)v[e], s);
  }
  return s;
}

__global__ void __launch_bounds__(kNormBlock)
grad_squares_kernel(const TensorChunk* __restrict__ list, int64_t chunks, double* __restrict__ partial) {
  __shared__ double s_wave[kNormWaves];
  double s = 0.0;
  for (int64_t i = blockIdx.x; i < chunks; i += gridDim.x) {
    const TensorChunk c = list[i];
    const int type = c.types & 255;
    ChunkData d;
    load_chunk(c, chunk_count(c), d);
    s += type == GBA_F32 ? chunk_squares<float>(d) : type == GBA_BF16 ? chunk_squares<bf16_t>(d) : chunk_squares<f16_t>(d);
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

template <typename T, typename O>
__device__ __forceinline__ void write_chunk(const ChunkData& d, O* __restrict__ out, int count, float coef) {
  constexpr int V = kVec<T>;
  const int units = count / V;
#pragma unroll
  for (int k = 0; k < kChunk / V / kNormBlock; ++k) {
    const int u = k * kNormBlock + threadIdx.x;
    float v[V];
    unpack<T>(d.unit[k], v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] *= coef;
    if (u < units) store_vec<O, V>(out + u * V, v);
  }
  const int left = units * V + threadIdx.x;
  if (left < count) out[left] = (O)(d.rest * coef);
}
template <typename T>
__device__ __forceinline__ void write_chunk(const ChunkData& d, const TensorChunk& c, int count, float coef) {
  const int type = c.types >> 8 & 255;
  if (type == GBA_F32) write_chunk<T>(d, static_cast<float*>(c.out), count, coef);
  else if (type == GBA_BF16) write_chunk<T>(d, static_cast<bf16_t*>(c.out), count, coef);
  else write_chunk<T>(d, static_cast<f16_t*>(c.out), count, coef);
}

// The chunks are taken from the last to the first: those that the sum read
// last are still in the caches.  A block asks for its first chunk before it
// adds up the partial sums.
__global__ void __launch_bounds__(kNormBlock)
clip_kernel(const TensorChunk* __restrict__ list, int64_t chunks, const double* __restrict__ partial, int blocks,
            double max_norm, float* __restrict__ norm, float* __restrict__ coef_out, int32_t* err) {
  __shared__ double s_wave[kNormWaves];
  float coef = 1.0f;
  bool known = false;
  for (int64_t i = blockIdx.x; i < chunks || !known; i += gridDim.x) {
    TensorChunk c{};
    int count = 0;
    ChunkData d;
    if (i < chunks) {
      c = list[chunks - 1 - i];
      if (c.out && !(known && coef == 1.0f && c.types >> 16)) {   // (in place with nothing to scale is skipped)
        count = chunk_count(c);
        load_chunk(c, count, d);
      }
    }
    if (!known) {
      known = true;
      const double n = sqrt(total_squares(partial, blocks, s_wave));
      const bool finite = isfinite(n);
      coef = !finite ? 0.0f : n > max_norm ? (float)(max_norm / n) : 1.0f;
      if (blockIdx.x == 0 && threadIdx.x == 0) {
        *norm = (float)n;
        if (coef_out) *coef_out = coef;
        if (!finite) raise_error(err, GBA_DERR_NONFINITE);
      }
      if (!finite) return;
      if (coef == 1.0f && c.types >> 16) count = 0;
    }
    if (count == 0) continue;
    const int type = c.types & 255;
    if (type == GBA_F32) write_chunk<float>(d, c, count, coef);
    else if (type == GBA_BF16) write_chunk<bf16_t>(d, c, count, coef);
    else write_chunk<f16_t>(d, c, count, coef);
  }
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
