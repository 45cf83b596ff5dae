// A gated linear recurrence over the positions of many sequences, column by
// column, and its gradient:
//   f = sigmoid(a),  h_t = f_t h_{t-1} + (1 - f_t) x_t;
//   g_t = dh_t + f_{t+1} g_{t+1},  dx_t = (1 - f_t) g_t,
//   da_t = g_t (h_{t-1} - x_t) f_t (1 - f_t),  dh0 = f_1 g_1.
//
// A step is the affine map h -> f h + (1 - f) x, and maps of consecutive steps
// make one map (F, S): h -> F h + S.  A tile of positions is held in registers
// from its only read to its only write: each lane group takes a few positions
// of its columns and makes their map, the maps are joined over the groups of
// the wave (shuffles) and over the waves (LDS), and every group then runs its
// own positions from the state that it enters with.  A sequence's first step
// takes the initial state instead of what comes before it, so the map of
// positions that hold a first step forgets the state (a flag, not F = 0: an
// infinity of one sequence stays there).  A block goes from tile to tile with
// the state.  The gradient is the same from the end to the front, its first
// steps the sequences' last ones.
//
// Blocks take whole sequences where there are enough of them.  Of few long
// ones each is cut into parts of equal length, the maps of all parts are made
// by a first launch, and each block of the second joins those before its own.
#include <algorithm>

#include "elements.hpp"
#include "gba_device.hpp"
#include "gba_internal.hpp"

namespace gba {

constexpr int kScanV = 4;                 // columns of a lane
constexpr int64_t kScanMaxParts = 512;    // most parts of the positions, times the groups of columns
constexpr int kScanMapBlock = 256;

__host__ __device__ static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

// ---------------------------------------------------------------- the gate
// The smaller of f and 1 - f, held with all its bits: t = 1 - f, or -f.
// (which of the two the sign bit says: either may be 0)
__device__ __forceinline__ float gate_of(float a) {
  // e^-|a| as a power of two; what its rounded exponent leaves out is put back as a factor near 1
  const float y = -1.44269504f * fabsf(a);
  const float rest = __builtin_fmaf(-1.44269504f, fabsf(a), -y) - 1.92596299e-8f * fabsf(a);
  float e = __builtin_amdgcn_exp2f(y);
  e = y > -126.0f ? __builtin_fmaf(e, 0.693147181f * rest, e) : e;   // (rest is not a number where a is infinite)
  return __builtin_copysignf(e * __builtin_amdgcn_rcpf(1.0f + e), a);
}
__device__ __forceinline__ bool gate_holds(float t) { return __float_as_int(t) >= 0; }
__device__ __forceinline__ float gate_f(float t) { return gate_holds(t) ? 1.0f - t : -t; }
__device__ __forceinline__ float gate_i(float t) { return gate_holds(t) ? t : 1.0f + t; }
// f h + (1 - f) x, one rounding beside that of the difference
__device__ __forceinline__ float gate_step(float t, float h, float x) {
  return __builtin_fmaf(t, x - h, gate_holds(t) ? h : x);
}
// f g
__device__ __forceinline__ float gate_back(float t, float g) { return __builtin_fmaf(-t, g, gate_holds(t) ? g : 0.0f); }

// ------------------------------------------------------ which sequence
// Packed sequences: the sequence of every position (-1 behind the last), and
// what an empty sequence hands on: its state, or its state's gradient.
struct ScanMapArgs {
  const int64_t* offsets;   // [B + 1]
  int32_t* seq;             // [n]
  const float* from;        // [B][D], may be null (0)
  float* to;                // [B][D], may be null
  int64_t n, B, D;
  int32_t* err;
};
__global__ void __launch_bounds__(kScanMapBlock)
scan_map_kernel(ScanMapArgs a) {
  const int64_t stride = (int64_t)gridDim.x * kScanMapBlock;
  const int64_t first = (int64_t)blockIdx.x * kScanMapBlock + threadIdx.x;
  for (int64_t p = first; p < a.n; p += stride) {
    int64_t lo = 0, hi = a.B;   // the last b with offsets[b] <= p, of lo .. hi - 1
    while (hi - lo > 1) {
      const int64_t mid = (lo + hi) >> 1;
      if (a.offsets[mid] <= p) lo = mid;
      else hi = mid;
    }
    a.seq[p] = a.offsets[lo] <= p && p < a.offsets[lo + 1] ? (int32_t)lo : -1;
  }
  for (int64_t b = first; b < a.B; b += stride)
    if (a.offsets[b] > a.offsets[b + 1] || (b == 0 && a.offsets[0] != 0) || a.offsets[b + 1] > a.n)
      raise_error(a.err, GBA_DERR_OFFSETS);
  if (!a.to) return;
  const int64_t waves = stride / kWave;
  for (int64_t b = first / kWave; b < a.B; b += waves) {
    if (a.offsets[b] < a.offsets[b + 1]) continue;
    for (int64_t c = lane_id(); c < a.D; c += kWave) a.to[b * a.D + c] = a.from ? a.from[b * a.D + c] : 0.0f;
  }
}

// ------------------------------------------------------------ the kernels
struct ScanArgs {
  RecurrenceArgs r;
  const int32_t* seq;      // packed: the sequence of each position; null: equal lengths
  int32_t length;          // ... of this many positions
  int32_t groups;          // of columns
  int32_t parts;           // of the sequences, or of the positions
  int32_t part_len;        // positions of a part; 0: parts are whole sequences
  float* part_F;           // [parts][D] the parts' maps
  float* part_S;
  int32_t* part_forget;    // [parts][groups]
  float* state;            // [B][D] copy of the states that sequences begin with, where a part writes over them
};

// One map over V columns.
struct Affine {
  float F[kScanV], S[kScanV];
  bool forget;             // the state before it does not matter
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < kScanV; ++e) {
      F[e] = 1.0f;
      S[e] = 0.0f;
    }
    forget = false;
  }
  // this after `before`
  __device__ __forceinline__ void after(const Affine& before) {
#pragma unroll
    for (int e = 0; e < kScanV; ++e) {
      S[e] = forget ? S[e] : __builtin_fmaf(F[e], before.S[e], S[e]);
      F[e] *= before.F[e];
    }
    forget |= before.forget;
  }
  __device__ __forceinline__ void apply(float (&h)[kScanV]) const {
#pragma unroll
    for (int e = 0; e < kScanV; ++e) h[e] = forget ? S[e] : __builtin_fmaf(F[e], h[e], S[e]);
  }
};

// How a tile lies over a block: LPC lanes over the columns of a group, SLOTS
// groups of lanes over the positions, T positions each.
template <int BLOCK, int LPC, int T>
struct ScanShape {
  static constexpr int WAVES = BLOCK / kWave;
  static constexpr int PER = kWave / LPC;       // slots of a wave
  static constexpr int SLOTS = BLOCK / LPC;
  static constexpr int TILE = SLOTS * T;
  static constexpr int COLUMNS = LPC * kScanV;
};

template <int BLOCK, int LPC, int T>
struct ScanShared {
  typedef ScanShape<BLOCK, LPC, T> Sh;
  float F[2][Sh::WAVES][Sh::COLUMNS], S[2][Sh::WAVES][Sh::COLUMNS];
  int forget[2][Sh::WAVES];
};

// Joins the slots' maps: leaves in `in` the state that this slot's positions
// are entered with and in `carry` (before: the tile's first) the state after the
// tile.  `waves`: how many of them hold positions.
template <int BLOCK, int LPC, int T, bool MAP>
__device__ __forceinline__ void scan_join(Affine& m, Affine& carry, float (&in)[kScanV], int waves, int& buffer,
                                          ScanShared<BLOCK, LPC, T>& s) {
  typedef ScanShape<BLOCK, LPC, T> Sh;
  const int lane = lane_id(), w = threadIdx.x / kWave, cl = lane % LPC;
  // inclusive over the slots of the wave
#pragma unroll
  for (int off = LPC; off < kWave; off <<= 1) {
    Affine b;
#pragma unroll
    for (int e = 0; e < kScanV; ++e) {
      b.F[e] = __shfl_up(m.F[e], off, kWave);
      b.S[e] = __shfl_up(m.S[e], off, kWave);
    }
    b.forget = __shfl_up((int)m.forget, off, kWave) != 0;
    if (lane >= off) m.after(b);
  }
  if (lane >= kWave - LPC) {
#pragma unroll
    for (int e = 0; e < kScanV; ++e) {
      s.F[buffer][w][cl * kScanV + e] = m.F[e];
      s.S[buffer][w][cl * kScanV + e] = m.S[e];
    }
    if (cl == 0) s.forget[buffer][w] = m.forget;   // (the first lane has columns, the last may have none)
  }
  __syncthreads();
  for (int k = 0; k < waves; ++k) {
    if (k == w) {
#pragma unroll
      for (int e = 0; e < kScanV; ++e) in[e] = carry.S[e];
    }
    Affine b;
#pragma unroll
    for (int e = 0; e < kScanV; ++e) {
      b.F[e] = s.F[buffer][k][cl * kScanV + e];
      b.S[e] = s.S[buffer][k][cl * kScanV + e];
    }
    b.forget = s.forget[buffer][k] != 0;
    if constexpr (MAP) {
      b.after(carry);
      carry = b;
    } else {
      b.apply(carry.S);
    }
  }
  buffer ^= 1;
  if constexpr (Sh::PER > 1 && !MAP) {
    // exclusive: what the slots before this one do
    Affine b;
#pragma unroll
    for (int e = 0; e < kScanV; ++e) {
      b.F[e] = __shfl_up(m.F[e], LPC, kWave);
      b.S[e] = __shfl_up(m.S[e], LPC, kWave);
    }
    b.forget = __shfl_up((int)m.forget, LPC, kWave) != 0;
    if (lane >= LPC) b.apply(in);
  }
}

// The state that part `part` of the positions is entered with (in carry.S):
// the maps of the `before` parts in front of it (front to back, or with BACK
// back to front), each wave a share of them.
template <int BLOCK, int LPC, int T, bool BACK>
__device__ __forceinline__ void enter_part(const ScanArgs& a, int part, int group, int c0, int count, Affine& carry,
                                           int& buffer, ScanShared<BLOCK, LPC, T>& s) {
  typedef ScanShape<BLOCK, LPC, T> Sh;
  const int before = BACK ? a.parts - 1 - part : part;
  const int w = threadIdx.x / kWave;
  const int lo = (int)((int64_t)before * w / Sh::WAVES), hi = (int)((int64_t)before * (w + 1) / Sh::WAVES);
  Affine m;
  m.clear();
  // (the lanes of a wave's first slot alone; the others hand on the identity)
  if (lane_id() < LPC) {
#pragma unroll 4
    for (int k = lo; k < hi; ++k) {
      const int j = BACK ? a.parts - 1 - k : k;
      Affine b;
      b.clear();
      if (count > 0) {
        load_part<float, kScanV>(a.part_F + (int64_t)j * a.r.D + c0, count, b.F);
        load_part<float, kScanV>(a.part_S + (int64_t)j * a.r.D + c0, count, b.S);
      }
      b.forget = a.part_forget[(int64_t)j * a.groups + group] != 0;
      b.after(m);
      m = b;
    }
  }
  float unused[kScanV];
  scan_join<BLOCK, LPC, T, false>(m, carry, unused, Sh::WAVES, buffer, s);
}

// The positions that a block takes.
__device__ __forceinline__ void part_range(const ScanArgs& a, int part, int64_t& p0, int64_t& p1) {
  const int64_t n = a.r.n, B = a.r.B;
  if (a.part_len) {
    p0 = (int64_t)part * a.part_len;
    p1 = p0 + a.part_len;
    int64_t end = n;
    if (a.seq) {
      end = a.r.offsets[B];
      end = end < 0 ? 0 : end > n ? n : end;
    }
    if (p1 > end) p1 = end;
    return;
  }
  const int64_t b0 = B * part / a.parts, b1 = B * (part + 1) / a.parts;
  if (a.seq) {
    p0 = a.r.offsets[b0];
    p1 = a.r.offsets[b1];
    p0 = p0 < 0 ? 0 : p0;
    p1 = p1 > n ? n : p1;
  } else {
    p0 = b0 * a.length;
    p1 = b1 * a.length;
  }
}

// Which of T positions from q on begin or end a sequence (bits), and the
// sequence of the first.
template <int T>
struct Bounds {
  uint32_t starts, ends;
  int32_t seq[T];
  __device__ __forceinline__ void find(const ScanArgs& a, int64_t q, int count) {
    starts = ends = 0;
    if (count <= 0) return;
    if (!a.seq) {
      int32_t b = (int32_t)((uint32_t)q / (uint32_t)a.length);
      int32_t r = (int32_t)q - b * a.length;
#pragma unroll
      for (int i = 0; i < T; ++i) {
        seq[i] = b;
        if (r == 0) starts |= 1u << i;
        if (r == a.length - 1) ends |= 1u << i;
        if (++r == a.length) {
          r = 0;
          ++b;
        }
      }
      return;
    }
    int32_t last = q > 0 ? a.seq[q - 1] : -2;   // (position 0 begins a sequence whatever the offsets)
    int32_t now = a.seq[q];
#pragma unroll
    for (int i = 0; i < T; ++i) {
      if (i < count) {
        const int32_t next = q + i + 1 < a.r.n ? a.seq[q + i + 1] : -1;
        seq[i] = now < 0 ? 0 : now;   // (offsets that are not in order alone have such positions)
        if (now != last) starts |= 1u << i;
        if (now != next) ends |= 1u << i;
        last = now;
        now = next;
      }
    }
  }
};

template <typename X, int BLOCK, int LPC, int T, bool MAP>
__global__ void __launch_bounds__(BLOCK)
scan_kernel(ScanArgs a) {
  typedef ScanShape<BLOCK, LPC, T> Sh;
  constexpr int V = kScanV;
  __shared__ ScanShared<BLOCK, LPC, T> s;
  const int group = (int)blockIdx.x % a.groups, part = (int)blockIdx.x / a.groups;
  const int slot = threadIdx.x / LPC, c0 = group * Sh::COLUMNS + (int)(threadIdx.x % LPC) * V;
  const int count = a.r.D - c0;   // columns of this lane, V of them or fewer (none: <= 0)
  const float* first_state = a.state && !MAP ? a.state : a.r.h0;
  int64_t p0, p1;
  part_range(a, part, p0, p1);
  int buffer = 0;
  Affine carry;
  carry.clear();
  if constexpr (!MAP)
    if (a.part_len && part > 0) enter_part<BLOCK, LPC, T, false>(a, part, group, c0, count, carry, buffer, s);
  for (int64_t p = p0; p < p1; p += Sh::TILE) {
    const int64_t q = p + slot * T;
    const int here = count <= 0 ? 0 : p1 - q < T ? (int)(p1 - q) : T;   // positions of this slot (none: <= 0)
    float t[T][V], x[T][V];
#pragma unroll
    for (int i = 0; i < T; ++i)
      if (i < here) {
        load_part<X, V>(static_cast<const X*>(a.r.x) + (q + i) * a.r.x_stride + c0, count, x[i]);
        load_part<X, V>(static_cast<const X*>(a.r.a) + (q + i) * a.r.a_stride + c0, count, t[i]);
      }
    Bounds<T> at;
    at.find(a, q, here);
    Affine m;
    m.clear();
#pragma unroll
    for (int i = 0; i < T; ++i) {
      if (i >= here) continue;
      const bool first = at.starts >> i & 1;
      float h0[V] = {};
      if (first && first_state) {
        load_part<float, V>(first_state + (int64_t)at.seq[i] * a.r.D + c0, count, h0);
        if (MAP && a.state) store_part<float, V>(a.state + (int64_t)at.seq[i] * a.r.D + c0, count, h0);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        t[i][e] = gate_of(t[i][e]);
        if (first) x[i][e] = gate_step(t[i][e], h0[e], x[i][e]);   // the state after the step
        m.S[e] = first ? x[i][e] : gate_step(t[i][e], m.S[e], x[i][e]);
        m.F[e] *= gate_f(t[i][e]);
      }
      m.forget |= first;
    }
    float h[V] = {};
    const int64_t rest = ceil_div(p1 - p, Sh::PER * T);
    scan_join<BLOCK, LPC, T, MAP>(m, carry, h, rest < Sh::WAVES ? (int)rest : Sh::WAVES, buffer, s);
    if constexpr (!MAP) {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (i >= here) continue;
        const bool first = at.starts >> i & 1;
#pragma unroll
        for (int e = 0; e < V; ++e) h[e] = first ? x[i][e] : gate_step(t[i][e], h[e], x[i][e]);
        store_part<X, V>(static_cast<X*>(a.r.h) + (q + i) * a.r.h_stride + c0, count, h);
        if (a.r.h_last && (at.ends >> i & 1))
          store_part<float, V>(a.r.h_last + (int64_t)at.seq[i] * a.r.D + c0, count, h);
      }
    }
  }
  if constexpr (MAP) {
    if ((int)threadIdx.x < LPC && count > 0) {
      store_part<float, V>(a.part_F + (int64_t)part * a.r.D + c0, count, carry.F);
      store_part<float, V>(a.part_S + (int64_t)part * a.r.D + c0, count, carry.S);
    }
    if (threadIdx.x == 0) a.part_forget[(int64_t)part * a.groups + group] = carry.forget;
  }
}

// The gradient: positions from the end; slot 0 takes a tile's last ones.  The
// state that runs through is f_t g_t, what a position hands to the one before it.
template <typename X, int BLOCK, int LPC, int T, bool MAP>
__global__ void __launch_bounds__(BLOCK)
scan_grad_kernel(ScanArgs a) {
  typedef ScanShape<BLOCK, LPC, T> Sh;
  constexpr int V = kScanV;
  __shared__ ScanShared<BLOCK, LPC, T> s;
  const int group = (int)blockIdx.x % a.groups, part = (int)blockIdx.x / a.groups;
  const int slot = threadIdx.x / LPC, c0 = group * Sh::COLUMNS + (int)(threadIdx.x % LPC) * V;
  const int count = a.r.D - c0;
  const float* last_grad = a.state && !MAP ? a.state : a.r.dh_last;
  int64_t p0, p1;
  part_range(a, part, p0, p1);
  int buffer = 0;
  Affine carry;
  carry.clear();
  if constexpr (!MAP)
    if (a.part_len && part + 1 < a.parts) enter_part<BLOCK, LPC, T, true>(a, part, group, c0, count, carry, buffer, s);
  for (int64_t p = p1; p > p0; p -= Sh::TILE) {
    const int64_t q = p - (int64_t)(slot + 1) * T;   // positions q .. q + T - 1, those from p0 on
    const int skip = q < p0 ? (p0 - q < T ? (int)(p0 - q) : T) : 0;
    const bool any = count > 0 && skip < T;
    float t[T][V], d[T][V], x[T][V], hp[T][V];
    Bounds<T> at;
    at.starts = at.ends = 0;
    if (any) {
      // (positions below p0, and below 0, are not of this slot)
      const int64_t q0 = q + skip;
      Bounds<T> b;
      b.find(a, q0, T - skip);
      at.starts = b.starts << skip;
      at.ends = b.ends << skip;
      // (the sequence of a position, as its place among the ones from q on)
#pragma unroll
      for (int i = 0; i < T; ++i) {
        at.seq[i] = 0;
#pragma unroll
        for (int j = 0; j <= i; ++j)
          if (i - j == skip) at.seq[i] = b.seq[j];
      }
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (i < skip) continue;
        const int64_t r = q + i;
        load_part<X, V>(static_cast<const X*>(a.r.dh) + r * a.r.dh_stride + c0, count, d[i]);
        load_part<X, V>(static_cast<const X*>(a.r.a) + r * a.r.a_stride + c0, count, t[i]);
        if constexpr (!MAP) {
          load_part<X, V>(static_cast<const X*>(a.r.x) + r * a.r.x_stride + c0, count, x[i]);
          if (!(at.starts >> i & 1)) {
            load_part<X, V>(static_cast<const X*>(a.r.h) + (r - 1) * a.r.h_stride + c0, count, hp[i]);
          } else if (a.r.h0) {
            load_part<float, V>(a.r.h0 + (int64_t)at.seq[i] * a.r.D + c0, count, hp[i]);
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e) hp[i][e] = 0.0f;
          }
        }
      }
    }
    Affine m;
    m.clear();
#pragma unroll
    for (int i = T - 1; i >= 0; --i) {
      if (!any || i < skip) continue;
      const bool last = at.ends >> i & 1;
      if (last && last_grad) {
        float g[V];
        load_part<float, V>(last_grad + (int64_t)at.seq[i] * a.r.D + c0, count, g);
        if (MAP && a.state) store_part<float, V>(a.state + (int64_t)at.seq[i] * a.r.D + c0, count, g);
#pragma unroll
        for (int e = 0; e < V; ++e) d[i][e] += g[e];
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        t[i][e] = gate_of(t[i][e]);
        m.S[e] = gate_back(t[i][e], last ? d[i][e] : d[i][e] + m.S[e]);
        m.F[e] *= gate_f(t[i][e]);
      }
      m.forget |= last;
    }
    float c[V] = {};
    const int64_t rest = ceil_div(p - p0, Sh::PER * T);
    scan_join<BLOCK, LPC, T, MAP>(m, carry, c, rest < Sh::WAVES ? (int)rest : Sh::WAVES, buffer, s);
    if constexpr (!MAP) {
#pragma unroll
      for (int i = T - 1; i >= 0; --i) {
        if (!any || i < skip) continue;
        const bool last = at.ends >> i & 1;
        float dx[V], da[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float g = last ? d[i][e] : d[i][e] + c[e];
          const float small = fabsf(t[i][e]);
          dx[e] = gate_i(t[i][e]) * g;
          da[e] = g * (hp[i][e] - x[i][e]) * (small * (1.0f - small));
          c[e] = gate_back(t[i][e], g);
        }
        store_part<X, V>(static_cast<X*>(a.r.dx) + (q + i) * a.r.dx_stride + c0, count, dx);
        store_part<X, V>(static_cast<X*>(a.r.da) + (q + i) * a.r.da_stride + c0, count, da);
        if (a.r.dh0 && (at.starts >> i & 1))
          store_part<float, V>(a.r.dh0 + (int64_t)at.seq[i] * a.r.D + c0, count, c);
      }
    }
  }
  if constexpr (MAP) {
    if ((int)threadIdx.x < LPC && count > 0) {
      store_part<float, V>(a.part_F + (int64_t)part * a.r.D + c0, count, carry.F);
      store_part<float, V>(a.part_S + (int64_t)part * a.r.D + c0, count, carry.S);
    }
    if (threadIdx.x == 0) a.part_forget[(int64_t)part * a.groups + group] = carry.forget;
  }
}

// ------------------------------------------------------------- launching
constexpr int kScanBlock = 512;
constexpr int kScanGradBlock = 512;
constexpr int64_t kScanSplitBelow = 128;   // blocks

// Lanes over the columns.
static int scan_lanes(int32_t D) {
  const int vecs = (int)std::min<int64_t>(ceil_div(D, kScanV), kWave);
  int l = 4;
  while (l < vecs) l *= 2;
  return l;
}
static int64_t scan_groups(int32_t D) { return ceil_div(D, (int64_t)scan_lanes(D) * kScanV); }
static int64_t scan_most_parts(int32_t D) { return std::max<int64_t>(1, kScanMaxParts / scan_groups(D)); }

// The sequence of each position, the parts' maps, and the states of as many
// sequences as are ever cut into parts.
struct ScanRoom {
  size_t seq, F, S, forget, state, bytes;
};
static ScanRoom scan_room(int64_t n, int64_t B, int32_t D) {
  ScanRoom r;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align_up(bytes);
    return here;
  };
  const int64_t parts = scan_most_parts(D), groups = scan_groups(D);
  r.seq = take((size_t)n * sizeof(int32_t));
  r.F = take((size_t)parts * D * sizeof(float));
  r.S = take((size_t)parts * D * sizeof(float));
  r.forget = take((size_t)parts * groups * sizeof(int32_t));
  r.state = take((size_t)std::min(B, kScanSplitBelow) * D * sizeof(float));
  r.bytes = at + 256;
  return r;
}
size_t recurrence_workspace_bytes(int64_t n, int64_t B, int32_t D) { return scan_room(n, B, D).bytes; }

template <typename X, int LPC, bool GRAD>
static hipError_t scan_in(ScanArgs a, void* ws, hipStream_t stream) {
  constexpr int BLOCK = GRAD ? kScanGradBlock : kScanBlock;
  constexpr int T = !GRAD && sizeof(X) == 2 ? 8 : 4;
  typedef ScanShape<BLOCK, LPC, T> Sh;
  const RecurrenceArgs& r = a.r;
  const int64_t tiles = ceil_div(r.n, Sh::TILE);
  a.groups = (int32_t)scan_groups(r.D);
  const ScanRoom room = scan_room(r.n, r.B, r.D);
  char* base = static_cast<char*>(ws);
  a.part_len = 0;
  a.parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>({r.B, tiles, 4096 / a.groups + 1}));
  const int64_t most = scan_most_parts(r.D);
  const bool split = r.B * a.groups < kScanSplitBelow && most > r.B && tiles > 2 * r.B;
  if (split) {
    const int64_t parts = std::min(most, tiles);
    a.part_len = (int32_t)(ceil_div(ceil_div(r.n, parts), Sh::TILE) * Sh::TILE);
    a.parts = (int32_t)ceil_div(r.n, a.part_len);
    a.part_F = reinterpret_cast<float*>(base + room.F);
    a.part_S = reinterpret_cast<float*>(base + room.S);
    a.part_forget = reinterpret_cast<int32_t*>(base + room.forget);
    if (GRAD ? r.dh_last && r.dh0 : r.h0 && r.h_last) a.state = reinterpret_cast<float*>(base + room.state);
  }
  const dim3 grid((unsigned)((int64_t)a.parts * a.groups));
  if constexpr (GRAD) {
    if (split) hipLaunchKernelGGL((scan_grad_kernel<X, BLOCK, LPC, T, true>), grid, dim3(BLOCK), 0, stream, a);
    hipLaunchKernelGGL((scan_grad_kernel<X, BLOCK, LPC, T, false>), grid, dim3(BLOCK), 0, stream, a);
  } else {
    if (split) hipLaunchKernelGGL((scan_kernel<X, BLOCK, LPC, T, true>), grid, dim3(BLOCK), 0, stream, a);
    hipLaunchKernelGGL((scan_kernel<X, BLOCK, LPC, T, false>), grid, dim3(BLOCK), 0, stream, a);
  }
  return hipGetLastError();
}

template <typename X, bool GRAD>
static hipError_t scan_as(const ScanArgs& a, void* ws, hipStream_t stream) {
  switch (scan_lanes(a.r.D)) {
    case 4: return scan_in<X, 4, GRAD>(a, ws, stream);
    case 8: return scan_in<X, 8, GRAD>(a, ws, stream);
    case 16: return scan_in<X, 16, GRAD>(a, ws, stream);
    case 32: return scan_in<X, 32, GRAD>(a, ws, stream);
    default: return scan_in<X, 64, GRAD>(a, ws, stream);
  }
}

template <bool GRAD>
static hipError_t launch_scan(const RecurrenceArgs& r, void* ws, int32_t* err, hipStream_t stream) {
  ScanArgs a{};
  a.r = r;
  if (r.offsets) {
    ScanMapArgs m;
    m.offsets = r.offsets;
    m.seq = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + scan_room(r.n, r.B, r.D).seq);
    m.from = GRAD ? r.dh_last : r.h0;
    m.to = GRAD ? r.dh0 : r.h_last;
    m.n = r.n;
    m.B = r.B;
    m.D = r.D;
    m.err = err;
    a.seq = m.seq;
    const int64_t work = std::max<int64_t>(r.n, m.to ? r.B * kWave : r.B);
    const int64_t blocks = std::min<int64_t>(ceil_div(work, kScanMapBlock), 1024);
    hipLaunchKernelGGL(scan_map_kernel, dim3((unsigned)blocks), dim3(kScanMapBlock), 0, stream, m);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  } else if (r.n > 0) {
    a.length = (int32_t)(r.n / r.B);
  }
  if (r.n == 0) return hipSuccess;
  if (r.type == GBA_F32) return scan_as<float, GRAD>(a, ws, stream);
  if (r.type == GBA_BF16) return scan_as<bf16_t, GRAD>(a, ws, stream);
  return scan_as<f16_t, GRAD>(a, ws, stream);
}

hipError_t launch_recurrence(const RecurrenceArgs& r, void* ws, int32_t* err, hipStream_t stream) {
  return launch_scan<false>(r, ws, err, stream);
}
hipError_t launch_recurrence_grad(const RecurrenceArgs& r, void* ws, int32_t* err, hipStream_t stream) {
  return launch_scan<true>(r, ws, err, stream);
}

}  // namespace gba
