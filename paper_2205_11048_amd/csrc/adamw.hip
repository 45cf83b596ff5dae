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
// and the element's place, so m and the root are right on average and the same
// call gives the same bits.  The step, a quotient of the two, is not: a root
// that became 0 beside an m that did not leaves it to eps (the largest step of
// gradients at 2^-18 of a block's largest of 1e-2, moments in 32 bits 1.2 lr: 13 lr at
// eps 1e-8, 4e4 at 1e-12, 0.9 at 2^-23, which is m's least code there).
//
// The list is cut into chunks of kAdamwChunk elements on the host, once, as the
// list of clipping is: a chunk's record holds all that a block needs.
//
// Bound by bytes: 16 M parameters with moments in 32 bits 72 us (417 MB, 5.8 TB/s),
// 200 M with moments in 8 bits, gradients and a copy in 16 565 us (3.2 GB, 5.7 TB/s),
// the moments read back 190 us each (1 GB).  Four elements of a thread and a block for each chunk:
// with sixteen of a thread the loads of a block wait for its arithmetic (830 us of the
// 200 M), with 4096 blocks that take chunks in turn 650.  Read and written past the
// caches: 16 M 94 us -> 82 (both with sixteen of a thread).
#include <algorithm>

#include "elements.hpp"
#include "gba_device.hpp"
#include "gba_internal.hpp"

namespace gba {

constexpr int kAdamBlock = 256;
constexpr int kAdamV = 4;                            // elements of a thread at a time: a wave takes one 8-bit block
constexpr int kMomentBlock = kWave * kAdamV;         // elements that share an exponent
static_assert(kMomentBlock == GBA_MOMENT_BLOCK, "a block of 8-bit moments is what a wave holds at a time");
constexpr int kAdamwChunk = kAdamBlock * kAdamV;
constexpr int64_t kAdamMaxBlocks = 1 << 17;

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

// The root of x >= 0, within an ulp, or EXACT: rounded to the nearest by one
// step of Newton's from the reciprocal root (the residue x - s^2 is exact in one
// fma).  The instructions do not know subnormal numbers: small x are scaled.
template <bool EXACT>
__device__ __forceinline__ float root_of(float x) {
  const bool small = x < 0x1p-96f;
  x *= small ? 0x1p64f : 1.0f;
  float s;
  if constexpr (EXACT) {
    const float y = __builtin_amdgcn_rsqf(fmaxf(x, 0x1p-126f));   // (0 stays 0)
    s = x * y;
    s = __builtin_fmaf(__builtin_fmaf(-s, s, x), 0.5f * y, s);
  } else {
    s = __builtin_amdgcn_sqrtf(x);
  }
  return s * (small ? 0x1p-32f : 1.0f);
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
constexpr uint32_t kInfinite = 0x7f800000u;   // magnitudes from here on are not finite

template <typename T, int V>
__device__ __forceinline__ void load_once(const T* __restrict__ p, int count, float (&o)[V]) {
  if (count >= V) {
    typedef typename VecOf<T, V>::type vec;
    const vec v = __builtin_nontemporal_load(reinterpret_cast<const vec*>(p));
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = (float)v[e];
  } else {
    load_part<T, V>(p, count, o);
  }
}

template <typename G, bool EIGHT>
__device__ __forceinline__ void adamw_chunk(const AdamwChunk& c, const AdamwStep& s, float coef, uint32_t key,
                                            int32_t* err) {
  constexpr int V = kAdamV;
  typedef uint8_t bytes __attribute__((ext_vector_type(V), aligned(1)));
  const int at = (int)threadIdx.x * V, left = c.count - at, block = at / kMomentBlock;
  float p[V] = {}, g[V] = {}, m[V] = {}, v[V] = {};
  bytes cm{}, cv{};
  int Em = 0, Ev = 0;
  if (left > 0) {
    load_once<float, V>(c.param + at, left, p);
    load_once<G, V>(static_cast<const G*>(c.grad) + at, left, g);
    if constexpr (!EIGHT) {
      load_once<float, V>(static_cast<const float*>(c.m) + at, left, m);
      load_once<float, V>(static_cast<const float*>(c.v) + at, left, v);
    } else {
      const uint8_t* a = static_cast<const uint8_t*>(c.m) + at;
      const uint8_t* b = static_cast<const uint8_t*>(c.v) + at;
      if (left >= V) {
        cm = *reinterpret_cast<const bytes*>(a);
        cv = *reinterpret_cast<const bytes*>(b);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          cm[e] = e < left ? a[e] : 0;
          cv[e] = e < left ? b[e] : 0;
        }
      }
      Em = c.m_exp[block];
      Ev = c.v_exp[block];
    }
  }
  const float keep = 1.0f - s.lr_wd * c.decay;
  float mn[V], vn[V], root[V], pn[V];
  uint32_t top_m = 0, top_v = 0;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if constexpr (EIGHT) {
      const float y = decode<3>(cm[e] & 127u, Em);
      m[e] = cm[e] & 128u ? -y : y;
      const float r = decode<4>(cv[e], Ev);
      v[e] = r * r;
    }
    const float x = g[e] * coef;
    mn[e] = s.b1 * m[e] + s.omb1 * x;
    vn[e] = s.b2 * v[e] + s.omb2 * (x * x);
    // (8 bits: the rounded root, which the code is of; else within an ulp)
    root[e] = root_of<EIGHT>(vn[e]);
    const float step = (s.lr_m * mn[e]) * __builtin_amdgcn_rcpf(root[e] * s.r_scale + s.eps);
    pn[e] = p[e] * keep - step;
    top_m = max(top_m, magnitude(mn[e]));
    top_v = max(top_v, magnitude(vn[e]));
  }
  if (max(top_m, top_v) >= kInfinite) {   // what is not finite stays as it was
    raise_error(err, GBA_DERR_NONFINITE);
    top_m = 0;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const bool fine = max(magnitude(mn[e]), magnitude(vn[e])) < kInfinite;
      mn[e] = fine ? mn[e] : m[e];
      vn[e] = fine ? vn[e] : v[e];
      pn[e] = fine ? pn[e] : p[e];
      root[e] = root_of<EIGHT>(vn[e]);
      top_m = max(top_m, magnitude(mn[e]));
    }
  }
  if constexpr (EIGHT) {
    const float top_r = fmaxf(fmaxf(root[0], root[1]), fmaxf(root[2], root[3]));
    Em = block_exponent<3>(wave_max(top_m));
    Ev = block_exponent<4>(wave_max(__float_as_uint(top_r)));
  }
  if (left <= 0) return;
  if constexpr (EIGHT) {
    const uint32_t here = mix_bits(key + c.block + (uint32_t)block);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const uint32_t random = mix_bits(here + (uint32_t)(at % kMomentBlock + e));
      cm[e] = (uint8_t)(encode<3>(fabsf(mn[e]), Em, random & 0xffffu) | (mn[e] < 0.0f ? 128u : 0u));
      cv[e] = (uint8_t)encode<4>(root[e], Ev, random >> 16);
    }
    uint8_t* a = static_cast<uint8_t*>(c.m) + at;
    uint8_t* b = static_cast<uint8_t*>(c.v) + at;
    if (left >= V) {
      *reinterpret_cast<bytes*>(a) = cm;
      *reinterpret_cast<bytes*>(b) = cv;
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e < left) {
          a[e] = cm[e];
          b[e] = cv[e];
        }
    }
    if (lane_id() == 0) {
      c.m_exp[block] = (uint8_t)Em;
      c.v_exp[block] = (uint8_t)Ev;
    }
  } else {
    store_part<float, V, true>(static_cast<float*>(c.m) + at, left, mn);
    store_part<float, V, true>(static_cast<float*>(c.v) + at, left, vn);
  }
  store_part<float, V, true>(c.param + at, left, pn);
  if (c.copy) store_part<V>(c.copy, c.types >> 8, at, left, pn);
}

__global__ void __launch_bounds__(kAdamBlock, 8)
adamw_kernel(const AdamwChunk* __restrict__ list, int64_t chunks, AdamwParams hp, AdamwStep s,
             const int64_t* __restrict__ t_device, int64_t t, uint32_t seed, const float* __restrict__ coef_device,
             int32_t* err) {
  const float coef = coef_device ? *coef_device : 1.0f;
  if (coef == 0.0f) return;   // the gradients' norm was not finite: no step
  if (t_device) {
    t = *t_device < 1 ? 1 : *t_device;   // also of what the rounding is drawn from
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
