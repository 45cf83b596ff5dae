// One AdamW step over many tensors (Loshchilov and Hutter 2019), element by
// element, with the moments in 32 bits or in 8:
//   g = coef * grad;  m' = b1 m + (1 - b1) g;  v' = b2 v + (1 - b2) g^2;
//   p' = (1 - lr wd) p - lr (m' / bc1) / (sqrt(v' / bc2) + eps).
//
// 8 bits: a block is 256 consecutive elements of a tensor, and what it holds
// of a moment is one power of two, 2^(E - 127), and a code per element that is
// a small float below it: 4 exponent bits and the mantissa, so a value keeps
// its relative precision over 15 binades below the block's largest and a whole
// block moves without its codes changing.  m takes a sign and 3 mantissa bits.
// Of v the root is held, in half as many binades, with 4.  A step moves a
// moment by far less than the distance of two codes (1 - b2 is 1/1000), which
// rounding to the nearest would lose every time: a code is rounded up with the
// probability of the fraction that it leaves, by a hash of the seed, the step
// and the element's place, so the moments are right on average and the same
// call gives the same bits.
//
// The list is cut into chunks of kAdamwChunk elements on the host, once, as the
// list of clipping is: a chunk's record holds all that a block needs.
#include <algorithm>

#include "elements.hpp"
#include "gba_device.hpp"
#include "gba_internal.hpp"

namespace gba {

constexpr int kAdamBlock = 256;
constexpr int kAdamV = 4;                            // elements of a thread at a time: a wave takes one 8-bit block
constexpr int kMomentBlock = kWave * kAdamV;         // elements that share an exponent
static_assert(kMomentBlock == GBA_MOMENT_BLOCK, "a block of 8-bit moments is what a wave holds at a time");
constexpr int kAdamVecs = 4;                         // vectors of a thread
constexpr int kAdamwChunk = kAdamBlock * kAdamV * kAdamVecs;
constexpr int64_t kAdamMaxBlocks = 2048;

struct AdamwChunk {
  float* param;        // the chunk's first element
  const void* grad;
  void* m;             // float, or a code per element
  void* v;
  uint8_t* m_exp;      // 8-bit moments: an exponent per block of them (null: moments in 32 bits)
  uint8_t* v_exp;
  void* copy;          // the updated parameters again, in copy_type (null: none)
  uint32_t tensor;     // the tensor's number in the list
  uint32_t block;      // the chunk's first block in its tensor
  float decay;         // the tensor's multiple of the weight decay
  int32_t count;       // elements of the chunk
  int32_t types;       // grad_type | copy_type << 8
  int32_t unused;
};
static_assert(sizeof(AdamwChunk) == 80, "the list's record");

static int size_of(int type) { return type == GBA_F32 ? 4 : 2; }

int64_t adamw_chunks(const gba_adamw_tensor* t, int32_t T) {
  int64_t c = 0;
  for (int32_t i = 0; i < T; ++i) c += (t[i].n + kAdamwChunk - 1) / kAdamwChunk;
  return c;
}
size_t adamw_list_bytes(int64_t chunks) { return (size_t)chunks * sizeof(AdamwChunk); }

void fill_adamw_list(const gba_adamw_tensor* t, int32_t T, void* list) {
  AdamwChunk* c = static_cast<AdamwChunk*>(list);
  for (int32_t i = 0; i < T; ++i) {
    const int moment = t[i].moment_bits / 8;
    for (int64_t at = 0; at < t[i].n; at += kAdamwChunk, ++c) {
      const int64_t block = at / kMomentBlock;
      c->param = t[i].param + at;
      c->grad = static_cast<const char*>(t[i].grad) + at * size_of(t[i].grad_type);
      c->m = static_cast<char*>(t[i].m) + at * moment;
      c->v = static_cast<char*>(t[i].v) + at * moment;
      c->m_exp = moment == 1 ? t[i].m_exp + block : nullptr;
      c->v_exp = moment == 1 ? t[i].v_exp + block : nullptr;
      c->copy = t[i].copy ? static_cast<char*>(t[i].copy) + at * size_of(t[i].copy_type) : nullptr;
      c->tensor = (uint32_t)i;
      c->block = (uint32_t)block;
      c->decay = (float)t[i].decay;
      c->count = (int32_t)std::min<int64_t>(kAdamwChunk, t[i].n - at);
      c->types = t[i].grad_type | t[i].copy_type << 8;
      c->unused = 0;
    }
  }
}

// The step's constants, from double.
struct AdamwStep {
  float b1, omb1, b2, omb2, eps;
  float lr_wd;     // lr * weight decay
  float lr_m;      // lr / bc1
  float r_scale;   // 1 / sqrt(bc2)
};

// b^t, t >= 1, by squaring: the host and the device, which reads t when it
// runs, then take the same constants.
__host__ __device__ inline double power_of(double b, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}
__host__ __device__ inline void bias_constants(const AdamwParams& p, int64_t t, AdamwStep& s) {
  if (t < 1) t = 1;
  s.lr_m = (float)(p.lr / (1.0 - power_of(p.beta1, t)));
  s.r_scale = (float)(1.0 / sqrt(1.0 - power_of(p.beta2, t)));
}

// 32 bits mixed by shifts and products with odd numbers (digits of e and of the golden ratio).
__device__ __forceinline__ uint32_t mix_bits(uint32_t x) {
  x ^= x >> 16;
  x *= 0xB7E15163u;
  x ^= x >> 15;
  x *= 0x9E3779B1u;
  return x ^ (x >> 16);
}

// The largest of x over the wave's lanes, in every lane.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
  const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
  return x > y ? x : y;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = dpp_max<0xB1>(x);    // lane ^ 1
  x = dpp_max<0x4E>(x);    // lane ^ 2
  x = dpp_max<0x141>(x);   // the other four of eight
  x = dpp_max<0x140>(x);   // the other eight of sixteen
  uint32_t y = (uint32_t)__shfl_xor((int)x, 16, kWave);
  x = x > y ? x : y;
  y = (uint32_t)__shfl_xor((int)x, 32, kWave);
  return x > y ? x : y;
}

// A code of MANT mantissa bits as a float's bits below 2^(E - 127): the code's
// exponent field is a float's with 112 taken off, codes below 2^MANT are a
// float's subnormals, and one ldexp puts the exponent right.
template <int MANT>
__device__ __forceinline__ float decode(uint32_t code, int E) {
  return ldexpf(__uint_as_float(code << (23 - MANT)), E - 15);
}
// ... and back, x >= 0 no more than the largest code: the bits that a code has
// no room for are the fraction to which 16 random bits (and a half of one) are added.
template <int MANT>
__device__ __forceinline__ uint32_t encode(float x, int E, uint32_t random) {
  constexpr int SHIFT = 23 - MANT;
  const uint32_t bits = __float_as_uint(ldexpf(x, 15 - E));
  const uint32_t code = (bits + (random << (SHIFT - 16)) + (1u << (SHIFT - 17))) >> SHIFT;
  constexpr uint32_t most = (1u << (4 + MANT)) - 1;
  return code < most ? code : most;
}
// E of a block whose largest value has these bits: the smallest with
// (2 - 2^-MANT) 2^(E - 127) no less.
template <int MANT>
__device__ __forceinline__ int block_exponent(uint32_t top) {
  const int E = (int)((top + ((1u << (23 - MANT)) - 1)) >> 23);
  return top == 0 ? 0 : E < 1 ? 1 : E > 254 ? 254 : E;
}

template <typename G, bool EIGHT>
__device__ __forceinline__ void adamw_chunk(const AdamwChunk& c, const AdamwStep& s, float coef, uint32_t key,
                                            int32_t* err) {
  constexpr int V = kAdamV, N = kAdamVecs;
  typedef uint8_t bytes __attribute__((ext_vector_type(V), aligned(1)));
  float p[N][V], g[N][V], m[N][V], v[N][V];
  int at[N], left[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    at[k] = (k * kAdamBlock + (int)threadIdx.x) * V;
    left[k] = c.count - at[k];
#pragma unroll
    for (int e = 0; e < V; ++e) p[k][e] = g[k][e] = m[k][e] = v[k][e] = 0.0f;
    if (left[k] <= 0) continue;
    load_part<float, V>(c.param + at[k], left[k], p[k]);
    load_part<G, V>(static_cast<const G*>(c.grad) + at[k], left[k], g[k]);
    if constexpr (!EIGHT) {
      load_part<float, V>(static_cast<const float*>(c.m) + at[k], left[k], m[k]);
      load_part<float, V>(static_cast<const float*>(c.v) + at[k], left[k], v[k]);
    }
  }
  if constexpr (EIGHT) {
    bytes cm[N], cv[N];
    int Em[N], Ev[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      cm[k] = cv[k] = bytes{};
      Em[k] = Ev[k] = 0;
      if (left[k] <= 0) continue;
      const uint8_t* a = static_cast<const uint8_t*>(c.m) + at[k];
      const uint8_t* b = static_cast<const uint8_t*>(c.v) + at[k];
      if (left[k] >= V) {
        cm[k] = *reinterpret_cast<const bytes*>(a);
        cv[k] = *reinterpret_cast<const bytes*>(b);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          cm[k][e] = e < left[k] ? a[e] : 0;
          cv[k][e] = e < left[k] ? b[e] : 0;
        }
      }
      Em[k] = c.m_exp[at[k] / kMomentBlock];
      Ev[k] = c.v_exp[at[k] / kMomentBlock];
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float x = decode<3>(cm[k][e] & 127u, Em[k]);
        m[k][e] = cm[k][e] & 128u ? -x : x;
        const float r = decode<4>(cv[k][e], Ev[k]);
        v[k][e] = r * r;
      }
  }
  const float keep = 1.0f - s.lr_wd * c.decay;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    float root[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float x = g[k][e] * coef;
      const float mn = s.b1 * m[k][e] + s.omb1 * x;
      const float vn = s.b2 * v[k][e] + s.omb2 * (x * x);
      const bool fine = isfinite(mn) && isfinite(vn);
      bad |= !fine;
      if (fine) {
        m[k][e] = mn;
        v[k][e] = vn;
      }
      // (8 bits: the rounded root, which the code is of; else within an ulp)
      root[e] = EIGHT ? sqrtf(v[k][e]) : __builtin_amdgcn_sqrtf(v[k][e]);
      const float step = (s.lr_m * mn) * __builtin_amdgcn_rcpf(root[e] * s.r_scale + s.eps);
      if (fine) p[k][e] = p[k][e] * keep - step;
    }
    if constexpr (EIGHT) {
      uint32_t top_m = 0, top_r = 0;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const uint32_t bm = __float_as_uint(m[k][e]) & 0x7fffffffu, br = __float_as_uint(root[e]);
        top_m = bm > top_m ? bm : top_m;
        top_r = br > top_r ? br : top_r;
      }
      const int Em = block_exponent<3>(wave_max(top_m)), Ev = block_exponent<4>(wave_max(top_r));
      if (left[k] <= 0) continue;
      const uint32_t here = mix_bits(key + c.block + (uint32_t)(at[k] / kMomentBlock));
      bytes cm, cv;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const uint32_t random = mix_bits(here + (uint32_t)(at[k] % kMomentBlock + e));
        cm[e] = (uint8_t)(encode<3>(fabsf(m[k][e]), Em, random & 0xffffu) | (m[k][e] < 0.0f ? 128u : 0u));
        cv[e] = (uint8_t)encode<4>(root[e], Ev, random >> 16);
      }
      uint8_t* a = static_cast<uint8_t*>(c.m) + at[k];
      uint8_t* b = static_cast<uint8_t*>(c.v) + at[k];
      if (left[k] >= V) {
        *reinterpret_cast<bytes*>(a) = cm;
        *reinterpret_cast<bytes*>(b) = cv;
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (e < left[k]) {
            a[e] = cm[e];
            b[e] = cv[e];
          }
      }
      if (lane_id() == 0) {
        c.m_exp[at[k] / kMomentBlock] = (uint8_t)Em;
        c.v_exp[at[k] / kMomentBlock] = (uint8_t)Ev;
      }
    }
    if (left[k] <= 0) continue;
    store_part<float, V>(c.param + at[k], left[k], p[k]);
    if constexpr (!EIGHT) {
      store_part<float, V>(static_cast<float*>(c.m) + at[k], left[k], m[k]);
      store_part<float, V>(static_cast<float*>(c.v) + at[k], left[k], v[k]);
    }
    if (c.copy) store_part<V>(c.copy, c.types >> 8, at[k], left[k], p[k]);
  }
  if (bad) raise_error(err, GBA_DERR_NONFINITE);
}

__global__ void __launch_bounds__(kAdamBlock)
adamw_kernel(const AdamwChunk* __restrict__ list, int64_t chunks, AdamwParams hp, AdamwStep s,
             const int64_t* __restrict__ t_device, int64_t t, uint32_t seed, const float* __restrict__ coef_device,
             int32_t* err) {
  const float coef = coef_device ? *coef_device : 1.0f;
  if (coef == 0.0f) return;   // the gradients' norm was not finite: no step
  if (t_device) {
    t = *t_device;
    bias_constants(hp, t, s);
  }
  const uint32_t step_key = mix_bits(seed + (uint32_t)t);
  for (int64_t i = blockIdx.x; i < chunks; i += gridDim.x) {
    const AdamwChunk c = list[i];
    const int type = c.types & 255;
    const uint32_t key = mix_bits(step_key + c.tensor);
    if (c.m_exp) {
      if (type == GBA_F32) adamw_chunk<float, true>(c, s, coef, key, err);
      else if (type == GBA_BF16) adamw_chunk<bf16_t, true>(c, s, coef, key, err);
      else adamw_chunk<f16_t, true>(c, s, coef, key, err);
    } else {
      if (type == GBA_F32) adamw_chunk<float, false>(c, s, coef, key, err);
      else if (type == GBA_BF16) adamw_chunk<bf16_t, false>(c, s, coef, key, err);
      else adamw_chunk<f16_t, false>(c, s, coef, key, err);
    }
  }
}

hipError_t launch_adamw(const void* list, int64_t chunks, const AdamwParams& hp, int64_t t, const int64_t* t_device,
                        uint32_t seed, const float* coef, int32_t* err, hipStream_t stream) {
  if (chunks == 0) return hipSuccess;
  AdamwStep s;
  s.b1 = (float)hp.beta1;
  s.omb1 = (float)(1.0 - hp.beta1);
  s.b2 = (float)hp.beta2;
  s.omb2 = (float)(1.0 - hp.beta2);
  s.eps = (float)hp.eps;
  s.lr_wd = (float)(hp.lr * hp.weight_decay);
  bias_constants(hp, t, s);
  hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)std::min(chunks, kAdamMaxBlocks)), dim3(kAdamBlock), 0, stream,
                     static_cast<const AdamwChunk*>(list), chunks, hp, s, t_device, t, seed, coef, err);
  return hipGetLastError();
}

// Four codes a thread; a wave takes a block of them.
template <int MANT>
__global__ void __launch_bounds__(kAdamBlock)
moments_read_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ exps, int64_t n,
                    float* __restrict__ out) {
  typedef uint8_t bytes __attribute__((ext_vector_type(kAdamV), aligned(1)));
  const int64_t step = (int64_t)gridDim.x * kAdamBlock * kAdamV;
  for (int64_t i = ((int64_t)blockIdx.x * kAdamBlock + threadIdx.x) * kAdamV; i < n; i += step) {
    const int count = n - i < kAdamV ? (int)(n - i) : kAdamV;
    const int E = exps[i / kMomentBlock];
    bytes c{};
    if (count == kAdamV) {
      c = *reinterpret_cast<const bytes*>(codes + i);
    } else {
#pragma unroll
      for (int e = 0; e < kAdamV; ++e) c[e] = e < count ? codes[i + e] : 0;
    }
    float v[kAdamV];
#pragma unroll
    for (int e = 0; e < kAdamV; ++e) {
      v[e] = decode<MANT>(MANT == 3 ? c[e] & 127u : c[e], E);
      if (MANT == 3 && c[e] & 128u) v[e] = -v[e];
    }
    store_part<float, kAdamV, true>(out + i, count, v);
  }
}

hipError_t launch_moments_read(const uint8_t* codes, const uint8_t* exps, int64_t n, int which, float* out,
                               hipStream_t stream) {
  if (n == 0) return hipSuccess;
  const int64_t blocks = std::min<int64_t>((n + kAdamBlock * kAdamV - 1) / (kAdamBlock * kAdamV), 1 << 20);
  if (which == GBA_MOMENT_M)
    hipLaunchKernelGGL(moments_read_kernel<3>, dim3((unsigned)blocks), dim3(kAdamBlock), 0, stream, codes, exps, n, out);
  else
    hipLaunchKernelGGL(moments_read_kernel<4>, dim3((unsigned)blocks), dim3(kAdamBlock), 0, stream, codes, exps, n, out);
  return hipGetLastError();
}

}  // namespace gba
