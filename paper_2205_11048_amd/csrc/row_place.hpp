// How the norms hold rows in registers: a row over the lanes of a wave or over
// several waves, and sums over it.
#pragma once

#include "elements.hpp"
#include "gba_device.hpp"

namespace gba {

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
// CHECK: every shape looks for narrow rows, not only the one that can have them
// (layer norm in half: how far the compiler joins products and conversions, and so
// the last bit, goes by it).
template <int V, int LPR, int NV, bool CHECK = true>
struct RowPlace {
  uint32_t col[NV];   // first column of each vector (unsigned: an offset from a uniform address)
  int shift;       // foreign elements of the last one
  bool last;       // the last one holds elements of this thread
  bool narrow;     // rows narrower than a vector (LPR = NV = 1): element by element
  int D;
  __device__ __forceinline__ RowPlace(int gl, int width) : D(width) {
    narrow = width < V;
#pragma unroll
    for (int k = 0; k < NV; ++k) col[k] = (uint32_t)((k * LPR + gl) * V);
    const int c = (int)col[NV - 1];
    last = c < width;
    const int moved = tiny() ? 0 : (c + V > width ? width - V : c);
    shift = c - moved < V ? c - moved : V;
    col[NV - 1] = (uint32_t)moved;
  }
  __device__ __forceinline__ bool tiny() const { return (CHECK || (LPR == 1 && NV == 1)) && narrow; }
  __device__ __forceinline__ bool own(int k, int e) const {
    return k + 1 < NV || (tiny() ? e < D : e >= shift);
  }
  template <typename P>
  __device__ __forceinline__ P* place(P* p, int k) const {
    return reinterpret_cast<P*>(const_cast<char*>(reinterpret_cast<const char*>(p)) + (uint32_t)(col[k] * (uint32_t)sizeof(P)));
  }
  template <typename P>
  __device__ __forceinline__ void load(const P* __restrict__ p, int k, float (&o)[V]) const {
    if (tiny()) load_part<P, V>(p, D, o);
    else load_vec<P, V>(place(p, k), o);
  }
  // as it is in memory
  template <typename T>
  __device__ __forceinline__ typename VecOf<T, V>::type load_raw(const T* __restrict__ p, int k) const {
    typename VecOf<T, V>::type v;
    if (tiny()) {
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = e < D ? p[e] : (T)0.0f;
    } else {
      v = *reinterpret_cast<const typename VecOf<T, V>::type*>(place(p, k));
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
  template <typename T>
  __device__ __forceinline__ void store(T* __restrict__ p, int k, const float (&o)[V]) const {
    if (tiny()) store_part<T, V>(p, D, o);
    else if (k + 1 < NV || last) store_vec<T, V, true>(place(p, k), o);
  }
  // foreign elements left out
  template <typename T>
  __device__ __forceinline__ void store_own(T* __restrict__ p, int k, const float (&o)[V]) const {
    if (tiny()) {
      store_part<T, V>(p, D, o);
    } else if (k + 1 < NV || shift == 0) {
      store_vec<T, V, true>(place(p, k), o);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e >= shift) p[col[k] + e] = (T)o[e];
    }
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

}  // namespace gba
