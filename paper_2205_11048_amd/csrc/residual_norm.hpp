// What the two directions of the norms with gate and residual share.
#pragma once

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

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

__device__ __forceinline__ float sigmoid(float a) { return 1.0f / (1.0f + expf(-a)); }
// f = sigmoid(a) and i = 1 - f, each within a few u of itself (f is 0 below -88.7): taken from a rounded f next to 1,
// i would be 6 % off at a = 16 and 0 from 17 on.
__device__ __forceinline__ void sigmoid_both(float a, float& f, float& i) {
  const float t = expf(-a);
  f = 1.0f / (1.0f + t);
  i = a < 0.0f ? 1.0f - f : t * f;   // (t may be infinite below 0)
}

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
    sigmoid_both(f[e], f[e], d[e]);
    d[e] *= f[e];
  }
}

// ------------------------------------------------------ rows in registers
constexpr int kRegBlock = 512;
constexpr int kWidest = 1024;             // most threads of a row
constexpr int kRegElements = 8;           // of a row, a thread's most
constexpr int kRegColumns = kWidest * kRegElements;
constexpr int64_t kRegBlocks = 2048;      // most blocks of a forward call

template <int VEC, int LPR, int NV>
struct NormShape {
  static constexpr int V = VEC;
  static constexpr int E = V * NV;
  static constexpr int BLOCK = LPR > kRegBlock ? LPR : kRegBlock;
  static constexpr int G = BLOCK / LPR;         // rows of a block at a time
  static constexpr int WAVES = BLOCK / kWave;
};

// Adds x over the wave, with every exchange an operand of the addition: the sum is in the last lane.
__device__ __forceinline__ float wave_total(float x) {
  x = lanes_sum<16>(x);
  // (lane 15 of rows 0 and 2 to rows 1 and 3, then lane 31 to rows 2 and 3)
  x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x142, 0xa, 0xf, false));
  x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x143, 0xc, 0xf, false));
  return x;
}
// As row_sum: rows of eight waves or more have their waves' sums added up by the
// lanes too (in turn they were 32 reads and additions of a thread at 16 waves).
template <int LPR, int WAVES, int N>
__device__ __forceinline__ void row_total(float (&x)[N], float (*s)[N][WAVES], int& buffer) {
  constexpr int PER = LPR / kWave;
  if constexpr (PER < 8) {
    row_sum<LPR, WAVES>(x, s, buffer);
  } else {
    static_assert(PER <= 16 && WAVES == PER, "one row of a block, its waves' sums in 16 lanes");
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = wave_total(x[i]);
    if (lane_id() == kWave - 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) s[buffer][i][threadIdx.x / kWave] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lanes_sum<PER>(s[buffer][i][lane_id() % PER]);
    buffer ^= 1;
  }
}

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
// The gate's row from element `from` on, as it is.
template <typename At, int NV, int V>
__device__ __forceinline__ void load_gate_row(const At& at, const void* gate, int type, int64_t from, float (&o)[NV][V]) {
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (type == GBA_F32) at.load(static_cast<const float*>(gate) + from, k, o[k]);
    else if (type == GBA_BF16) at.load(static_cast<const bf16_t*>(gate) + from, k, o[k]);
    else at.load(static_cast<const f16_t*>(gate) + from, k, o[k]);
  }
}
template <int NV, int V>
__device__ __forceinline__ void gate_factors(int kind, float (&f)[NV][V]) {
  if (kind != GBA_GATE_SIGMOID) return;
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < V; ++e) f[k][e] = sigmoid(f[k][e]);
}
// Calls f.run<stream's type, the others' type>().
template <typename F>
static hipError_t with_types(const Args& a, const F& f) {
  if (a.type == GBA_F32) return f.template run<float, float>();
  if (a.type == GBA_BF16) return a.stream_type == GBA_F32 ? f.template run<float, bf16_t>() : f.template run<bf16_t, bf16_t>();
  return a.stream_type == GBA_F32 ? f.template run<float, f16_t>() : f.template run<f16_t, f16_t>();
}
}  // namespace gba
