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
// the state, and loads the next tile before it joins the maps of this one.
// The gradient is the same from the end to the front, its first steps the
// sequences' last ones.
//
// Blocks take whole sequences where there are enough of them.  Of few long
// ones each is cut into parts of equal length, the maps of all parts are made
// by a first launch, and each block of the second joins those before its own.
#include <algorithm>

#include "elements.hpp"
#include "gba_device.hpp"
#include "gba_internal.hpp"

namespace gba {

constexpr int kScanBlock = 256;
constexpr int kScanWaves = kScanBlock / kWave;
constexpr int kScanV = 4;                  // columns of a lane
constexpr int kScanLanes = 32;             // most lanes over the columns of a block
constexpr int kScanWidest = kScanLanes * kScanV;
constexpr int kScanSimd = 2;               // waves of a SIMD that the registers are for
constexpr int64_t kScanBlocks = 256 * kScanSimd;   // ... and so the blocks of a round, a wave of each on every SIMD
constexpr int64_t kScanSplitBelow = 192;   // blocks

__host__ __device__ static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

// ---------------------------------------------------------------- the gate
// f = sigmoid(a) and i = 1 - f, each within a few u of itself, or (not FINE:
// 16-bit types, whose values carry 2^-9 or 2^-12 anyway) |a| u more.
template <bool FINE>
__device__ __forceinline__ void gate_of(float a, float& f, float& i) {
  const float y = -1.44269504f * fabsf(a);
  float e = __builtin_amdgcn_exp2f(y);
  if constexpr (FINE) {   // what y's rounding leaves out is put back as a factor near 1
    const float rest = __builtin_fmaf(-1.92596299e-8f, fabsf(a), __builtin_fmaf(-1.44269504f, fabsf(a), -y));
    e = y > -126.0f ? __builtin_fmaf(e, 0.693147181f * rest, e) : e;   // (rest is not a number where a is infinite)
  }
  const float big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
  const bool holds = a >= 0.0f;
  f = holds ? big : small;
  i = holds ? small : big;
}

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
__global__ void __launch_bounds__(kScanBlock)
scan_map_kernel(ScanMapArgs a) {
  const int64_t stride = (int64_t)gridDim.x * kScanBlock;
  const int64_t first = (int64_t)blockIdx.x * kScanBlock + threadIdx.x;
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
  int32_t parts;           // of the positions
  int32_t part_len;        // positions of a part
  bool split;              // parts are cut through sequences
  float* part_F;           // [parts][D] the parts' maps
  float* part_S;
  int32_t* part_forget;    // [parts][groups]
  float* state;            // [B][D] copy of the states that sequences begin with, where a part writes over them
};

// One map over V columns.
template <int V>
struct Affine {
  float F[V], S[V];
  bool forget;             // the state before it does not matter
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      F[e] = 1.0f;
      S[e] = 0.0f;
    }
    forget = false;
  }
  // this after `before`
  __device__ __forceinline__ void after(const Affine& before) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      S[e] = forget ? S[e] : __builtin_fmaf(F[e], before.S[e], S[e]);
      F[e] *= before.F[e];
    }
    forget |= before.forget;
  }
  __device__ __forceinline__ void apply(float (&h)[V]) const {
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = forget ? S[e] : __builtin_fmaf(F[e], h[e], S[e]);
  }
};

// Positions of a lane.
template <bool GRAD>
constexpr int kScanT = GRAD ? 4 : 8;

// How a tile lies over a block: LPC lanes with V columns each over the columns
// of a group, SLOTS groups of lanes over the positions, T positions each.
template <int LPC, int V, int T>
struct ScanShape {
  static constexpr int PER = kWave / LPC;       // slots of a wave
  static constexpr int SLOTS = kScanBlock / LPC;
  static constexpr int TILE = SLOTS * T;
  static constexpr int COLUMNS = LPC * V;
};

// A lane's columns.  The last lane's are moved back to end at the row's end:
// its first `shift` columns are other lanes' (all V past the end), which it
// computes as they do and does not store.
template <int V>
struct ScanColumns {
  int at, shift;
  __device__ __forceinline__ ScanColumns(int c, int D) {
    at = c + V > D ? D - V : c;
    shift = c - at < V ? c - at : V;
  }
  // p: the lane's first column
  template <typename X>
  __device__ __forceinline__ void store(X* __restrict__ p, const float (&o)[V]) const {
    if (shift == 0) {
      store_vec<X, V, true>(p, o);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e >= shift) p[e] = (X)o[e];
    }
  }
};

template <int LPC, int V>
struct ScanShared {
  float F[2][kScanWaves][LPC * V], S[2][kScanWaves][LPC * V];
  int forget[2][kScanWaves];
};

// Joins the slots' maps: leaves in `in` the state that this slot's positions
// are entered with and in `carry` (before: the tile's first) the state after the
// tile.
template <int LPC, int V, bool MAP>
__device__ __forceinline__ void scan_join(Affine<V>& m, Affine<V>& carry, float (&in)[V], int& buffer,
                                          ScanShared<LPC, V>& s) {
  const int lane = lane_id(), w = threadIdx.x / kWave, cl = lane % LPC;
  // inclusive over the slots of the wave
#pragma unroll
  for (int off = LPC; off < kWave; off <<= 1) {
    Affine<V> b;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      b.F[e] = __shfl_up(m.F[e], off, kWave);
      b.S[e] = __shfl_up(m.S[e], off, kWave);
    }
    b.forget = __shfl_up((int)m.forget, off, kWave) != 0;
    if (lane >= off) m.after(b);
  }
  if (lane >= kWave - LPC) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      s.F[buffer][w][cl * V + e] = m.F[e];
      s.S[buffer][w][cl * V + e] = m.S[e];
    }
    if (cl == 0) s.forget[buffer][w] = m.forget;
  }
  // exclusive: what the slots before this one do
  Affine<V> x;
  if constexpr (!MAP) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      x.F[e] = __shfl_up(m.F[e], LPC, kWave);
      x.S[e] = __shfl_up(m.S[e], LPC, kWave);
    }
    x.forget = __shfl_up((int)m.forget, LPC, kWave) != 0;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kScanWaves; ++k) {
    if (k == w) {
#pragma unroll
      for (int e = 0; e < V; ++e) in[e] = carry.S[e];
    }
    Affine<V> b;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      b.F[e] = s.F[buffer][k][cl * V + e];
      b.S[e] = s.S[buffer][k][cl * V + e];
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
  if constexpr (!MAP)
    if (lane >= LPC) x.apply(in);
}

// The state that part `part` of the positions is entered with (in carry.S):
// the maps of the parts in front of it (front to back, or with BACK back to
// front), each slot a share of them.
template <int LPC, int V, bool BACK>
__device__ __forceinline__ void enter_part(const ScanArgs& a, int part, int group, int col, Affine<V>& carry, int& buffer,
                                           ScanShared<LPC, V>& s) {
  constexpr int SLOTS = kScanBlock / LPC;
  const int before = BACK ? a.parts - 1 - part : part;
  const int slot = threadIdx.x / LPC;
  const int lo = (int)((int64_t)before * slot / SLOTS), hi = (int)((int64_t)before * (slot + 1) / SLOTS);
  Affine<V> m;
  m.clear();
#pragma unroll 4
  for (int k = lo; k < hi; ++k) {
    const int j = BACK ? a.parts - 1 - k : k;
    Affine<V> b;
    load_vec<float, V>(a.part_F + (int64_t)j * a.r.D + col, b.F);
    load_vec<float, V>(a.part_S + (int64_t)j * a.r.D + col, b.S);
    b.forget = a.part_forget[(int64_t)j * a.groups + group] != 0;
    b.after(m);
    m = b;
  }
  float unused[V];
  scan_join<LPC, V, false>(m, carry, unused, buffer, s);
}

// Where the first sequence that begins at position p or behind it begins.
__device__ __forceinline__ int64_t next_start(const ScanArgs& a, int64_t p) {
  if (p <= 0 || p >= a.r.n) return p <= 0 ? 0 : a.r.n;
  const int32_t here = a.seq[p];
  if (here != a.seq[p - 1]) return p;
  if (here < 0) return a.r.n;
  const int64_t end = a.r.offsets[here + 1];
  return end < a.r.n ? end : a.r.n;   // (behind p, whatever the offsets)
}

// Where a block is in the order of parts and groups: blocks go to the eight dies
// in turn, and neighbours, which read the same rows, come to one die.
__device__ __forceinline__ unsigned block_place() {
  constexpr unsigned kDies = 8;
  const unsigned n = gridDim.x, each = n / kDies, more = n % kDies, die = blockIdx.x % kDies;
  return die * each + (die < more ? die : more) + blockIdx.x / kDies;
}

// The positions that a block takes.
__device__ __forceinline__ void part_range(const ScanArgs& a, int part, int64_t& p0, int64_t& p1) {
  p0 = (int64_t)part * a.part_len;
  p1 = p0 + a.part_len;
  int64_t end = a.r.n;
  if (a.seq) {
    if (!a.split) {
      p0 = next_start(a, p0);
      p1 = next_start(a, p1);
    }
    end = a.r.offsets[a.r.B];
    end = end < 0 ? 0 : end > a.r.n ? a.r.n : end;
  }
  if (p1 > end) p1 = end;
  p0 = __builtin_amdgcn_readfirstlane((int)p0);   // (the same in every lane, also to the compiler)
  p1 = __builtin_amdgcn_readfirstlane((int)p1);
}

// Which of T positions from q on begin and end a sequence, as bits.
template <int T>
struct Bounds {
  uint32_t starts, ends;
  int32_t seq[T + 2];      // packed: the sequences of the position before, of the T and of the one behind
  // (positions below 0 and from n on are not looked at by `find`)
  __device__ __forceinline__ void load(const ScanArgs& a, int64_t q) {
    if (!a.seq) return;
    const int64_t last = a.r.n - 1;
    if (q >= 1 && q + T <= last) {
#pragma unroll
      for (int i = 0; i < T + 2; ++i) seq[i] = a.seq[q - 1 + i];
    } else {
#pragma unroll
      for (int i = 0; i < T + 2; ++i) {
        const int64_t p = q - 1 + i;
        seq[i] = a.seq[p < 0 ? 0 : p > last ? last : p];
        if (p < 0 || p > last) seq[i] = -2;   // (position 0 begins a sequence whatever the offsets)
      }
    }
  }
  // of positions q + from .. q + to - 1
  __device__ __forceinline__ void find(const ScanArgs& a, int64_t q, int from, int to) {
    starts = ends = 0;
    if (a.seq) {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (seq[i + 1] != seq[i]) starts |= 1u << i;
        if (seq[i + 1] != seq[i + 2]) ends |= 1u << i;
      }
    } else {
      const int32_t p = (int32_t)(q < 0 ? 0 : q);   // (only those below 0 are wrong, and masked)
      int32_t r = p - (int32_t)((uint32_t)p / (uint32_t)a.length) * a.length - (int32_t)(p - q);
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (r == 0) starts |= 1u << i;
        if (r == a.length - 1) ends |= 1u << i;
        r = r == a.length - 1 ? 0 : r + 1;
      }
    }
    const uint32_t mask = (to <= 0 ? 0u : (1u << to) - 1) & ~((1u << from) - 1);
    starts &= mask;
    ends &= mask;
  }
  static __device__ __forceinline__ int64_t sequence(const ScanArgs& a, int64_t p) {
    if (!a.seq) return (uint32_t)p / (uint32_t)a.length;
    const int32_t b = a.seq[p];
    return b < 0 ? 0 : b;   // (offsets that are not in order alone have such positions)
  }
};

// A lane's place in a matrix, in bytes from a tile's first row: `slot` and
// column.  The rows of a tile are then at a uniform address each, to which this
// is added (the compiler would otherwise hold a pointer per row and matrix in
// registers, twice as many as the tile itself takes).
template <typename X>
__device__ __forceinline__ uint64_t lane_place(int64_t stride, int64_t row, int col) {
  return (uint64_t)(row * stride + col) * sizeof(X);
}
__device__ __forceinline__ void keep_place(uint64_t& place) { asm volatile("" : "+v"(place)); }

// A matrix's rows from a uniform one on.
template <typename X>
struct RowsFrom {
  char* first;
  int64_t step;   // bytes
  __device__ __forceinline__ RowsFrom(const void* base, int64_t stride, int64_t row)
      : first(const_cast<char*>(static_cast<const char*>(base)) + row * stride * (int64_t)sizeof(X)),
        step(stride * (int64_t)sizeof(X)) {}
  __device__ __forceinline__ X* at(int i, uint64_t place) const {
    return reinterpret_cast<X*>(first + i * step + place);
  }
  template <int V>
  __device__ __forceinline__ typename VecOf<X, V>::type load(int i, uint64_t place) const {
    typedef typename VecOf<X, V>::type vec;
    return __builtin_nontemporal_load(reinterpret_cast<const vec*>(at(i, place)));
  }
};

template <typename X, int LPC, int V, int T, bool MAP>
__global__ void __launch_bounds__(kScanBlock, kScanSimd)
scan_kernel(ScanArgs a) {
  typedef ScanShape<LPC, V, T> Sh;
  typedef typename VecOf<X, V>::type vec;
  __shared__ ScanShared<LPC, V> s;
  const unsigned block = block_place();
  const int group = (int)(block % (unsigned)a.groups), part = (int)(block / (unsigned)a.groups);
  const int slot = threadIdx.x / LPC;
  const ScanColumns<V> col(group * Sh::COLUMNS + (int)(threadIdx.x % LPC) * V, a.r.D);
  const float* first_state = a.state && !MAP ? a.state : a.r.h0;
  int64_t p0, p1;
  part_range(a, part, p0, p1);
  int buffer = 0;
  Affine<V> carry;
  carry.clear();
  vec x[T] = {}, g[T] = {};
  Bounds<T> at;
  uint64_t place_x = lane_place<X>(a.r.x_stride, slot * T, col.at), place_a = lane_place<X>(a.r.a_stride, slot * T, col.at);
  uint64_t place_h = lane_place<X>(a.r.h_stride, slot * T, col.at);
  auto load = [&](int64_t p) {
    keep_place(place_x);
    keep_place(place_a);
    const int64_t q = p + slot * T;
    const RowsFrom<X> rows_a(a.r.a, a.r.a_stride, p), rows_x(a.r.x, a.r.x_stride, p);
    if (p + Sh::TILE <= p1) {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        g[i] = rows_a.template load<V>(i, place_a);
        x[i] = rows_x.template load<V>(i, place_x);
      }
    } else {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (q + i >= p1) continue;
        g[i] = rows_a.template load<V>(i, place_a);
        x[i] = rows_x.template load<V>(i, place_x);
      }
    }
    at.load(a, q);
  };
  if (p0 < p1) load(p0);
  if constexpr (!MAP)
    if (a.split && part > 0) enter_part<LPC, V, false>(a, part, group, col.at, carry, buffer, s);
  for (int64_t p = p0; p < p1; p += Sh::TILE) {
    const int64_t q = p + slot * T;
    const int here = p1 - q < T ? (int)(p1 - q) : T;   // positions of this slot (none: <= 0)
    float f[T][V], v[T][V];
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        gate_of<sizeof(X) == 4>((float)g[i][e], f[i][e], v[i][e]);
        v[i][e] *= (float)x[i][e];
      }
    // (what slots past the end compute goes nowhere: the tile is the last, and nobody enters with the last part's map)
    at.find(a, q, 0, here);
    const uint32_t starts = at.starts, ends = at.ends;
    if (starts && first_state) {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (!(starts >> i & 1)) continue;
        const int64_t to = Bounds<T>::sequence(a, q + i) * a.r.D;
        float h0[V];
        load_vec<float, V>(first_state + to + col.at, h0);
        if (MAP && a.state) col.store(a.state + to + col.at, h0);
#pragma unroll
        for (int e = 0; e < V; ++e) v[i][e] = __builtin_fmaf(f[i][e], h0[e], v[i][e]);   // the state after the step
      }
    }
    if (p + Sh::TILE < p1) load(p + Sh::TILE);
    Affine<V> m;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      m.F[e] = f[0][e];
      m.S[e] = v[0][e];
    }
#pragma unroll
    for (int i = 1; i < T; ++i) {
      const bool first = starts >> i & 1;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        m.S[e] = first ? v[i][e] : __builtin_fmaf(f[i][e], m.S[e], v[i][e]);
        m.F[e] *= f[i][e];
      }
    }
    m.forget = starts != 0;
    float h[V];
    scan_join<LPC, V, MAP>(m, carry, h, buffer, s);
    if constexpr (!MAP) {
      keep_place(place_h);
      const RowsFrom<X> out(a.r.h, a.r.h_stride, p);
#pragma unroll
      for (int i = 0; i < T; ++i) {
        const bool first = starts >> i & 1;
#pragma unroll
        for (int e = 0; e < V; ++e) h[e] = first ? v[i][e] : __builtin_fmaf(f[i][e], h[e], v[i][e]);
        if (i < here) col.store(out.at(i, place_h), h);
        if (a.r.h_last && (ends >> i & 1)) col.store(a.r.h_last + Bounds<T>::sequence(a, q + i) * a.r.D + col.at, h);
      }
    }
  }
  if constexpr (MAP) {
    if ((int)threadIdx.x < LPC) {
      store_vec<float, V>(a.part_F + (int64_t)part * a.r.D + col.at, carry.F);
      store_vec<float, V>(a.part_S + (int64_t)part * a.r.D + col.at, carry.S);
    }
    if (threadIdx.x == 0) a.part_forget[(int64_t)part * a.groups + group] = carry.forget;
  }
}

// The gradient: positions from the end; slot 0 takes a tile's last ones.  The
// state that runs through is f_t g_t, what a position hands to the one before it.
template <typename X, int LPC, int V, int T, bool MAP>
__global__ void __launch_bounds__(kScanBlock, kScanSimd)
scan_grad_kernel(ScanArgs a) {
  typedef ScanShape<LPC, V, T> Sh;
  typedef typename VecOf<X, V>::type vec;
  __shared__ ScanShared<LPC, V> s;
  const unsigned block = block_place();
  const int group = (int)(block % (unsigned)a.groups), part = (int)(block / (unsigned)a.groups);
  const int slot = threadIdx.x / LPC;
  const ScanColumns<V> col(group * Sh::COLUMNS + (int)(threadIdx.x % LPC) * V, a.r.D);
  const float* last_grad = a.state && !MAP ? a.state : a.r.dh_last;
  int64_t p0, p1;
  part_range(a, part, p0, p1);
  int buffer = 0;
  Affine<V> carry;
  carry.clear();
  vec gate[T] = {}, dh[T] = {}, x[T] = {}, before[T] = {};
  Bounds<T> at;
  // (a tile's last slot is its first one in memory)
  const int back = (Sh::SLOTS - 1 - slot) * T;
  uint64_t place_a = lane_place<X>(a.r.a_stride, back, col.at), place_d = lane_place<X>(a.r.dh_stride, back, col.at);
  uint64_t place_x = lane_place<X>(a.r.x_stride, back, col.at), place_h = lane_place<X>(a.r.h_stride, back, col.at);
  uint64_t place_dx = lane_place<X>(a.r.dx_stride, back, col.at), place_da = lane_place<X>(a.r.da_stride, back, col.at);
  auto load = [&](int64_t p) {   // positions p - TILE .. p - 1, those from p0 on
    keep_place(place_a);
    keep_place(place_d);
    keep_place(place_x);
    keep_place(place_h);
    const int64_t first = p - Sh::TILE, q = first + back;
    const RowsFrom<X> rows_a(a.r.a, a.r.a_stride, first), rows_d(a.r.dh, a.r.dh_stride, first);
    const RowsFrom<X> rows_x(a.r.x, a.r.x_stride, first), rows_h(a.r.h, a.r.h_stride, first - 1);
    if (first >= p0 && first > 0) {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        gate[i] = rows_a.template load<V>(i, place_a);
        dh[i] = rows_d.template load<V>(i, place_d);
        if constexpr (!MAP) {
          x[i] = rows_x.template load<V>(i, place_x);
          before[i] = rows_h.template load<V>(i, place_h);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (q + i < p0) continue;
        gate[i] = rows_a.template load<V>(i, place_a);
        dh[i] = rows_d.template load<V>(i, place_d);
        if constexpr (!MAP) {
          x[i] = rows_x.template load<V>(i, place_x);
          if (q + i > 0) before[i] = rows_h.template load<V>(i, place_h);
        }
      }
    }
    at.load(a, q);
  };
  if (p0 < p1) load(p1);
  if constexpr (!MAP)
    if (a.split && part + 1 < a.parts) enter_part<LPC, V, true>(a, part, group, col.at, carry, buffer, s);
  for (int64_t p = p1; p > p0; p -= Sh::TILE) {
    const int64_t q = p - Sh::TILE + back;
    const int skip = q < p0 ? (p0 - q < T ? (int)(p0 - q) : T) : 0;
    float f[T][V], in[T][V], d[T][V], diff[T][V];
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        gate_of<sizeof(X) == 4>((float)gate[i][e], f[i][e], in[i][e]);
        d[i][e] = (float)dh[i][e];
        if constexpr (!MAP) diff[i][e] = (float)before[i][e] - (float)x[i][e];
      }
    if (MAP && p - Sh::TILE < p0) {   // in front of the part (of a map, which is handed on): steps that do nothing
#pragma unroll
      for (int i = 0; i < T; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          f[i][e] = i < skip ? 1.0f : f[i][e];
          d[i][e] = i < skip ? 0.0f : d[i][e];
        }
    }
    at.find(a, q, skip, T);
    const uint32_t starts = at.starts, ends = at.ends;
    if (starts && !MAP) {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (!(starts >> i & 1)) continue;
        float h0[V] = {};
        if (a.r.h0) load_vec<float, V>(a.r.h0 + Bounds<T>::sequence(a, q + i) * a.r.D + col.at, h0);
#pragma unroll
        for (int e = 0; e < V; ++e) diff[i][e] = h0[e] - (float)x[i][e];
      }
    }
    if (ends && last_grad) {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (!(ends >> i & 1)) continue;
        const int64_t to = Bounds<T>::sequence(a, q + i) * a.r.D;
        float g[V];
        load_vec<float, V>(last_grad + to + col.at, g);
        if (MAP && a.state) col.store(a.state + to + col.at, g);
#pragma unroll
        for (int e = 0; e < V; ++e) d[i][e] += g[e];
      }
    }
    if (p - Sh::TILE > p0) load(p - Sh::TILE);
    Affine<V> m;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      m.F[e] = f[T - 1][e];
      m.S[e] = f[T - 1][e] * d[T - 1][e];
    }
#pragma unroll
    for (int i = T - 2; i >= 0; --i) {
      const bool last = ends >> i & 1;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        m.S[e] = f[i][e] * (last ? d[i][e] : d[i][e] + m.S[e]);
        m.F[e] *= f[i][e];
      }
    }
    m.forget = ends != 0;
    float c[V];
    scan_join<LPC, V, MAP>(m, carry, c, buffer, s);
    if constexpr (!MAP) {
      keep_place(place_dx);
      keep_place(place_da);
      const RowsFrom<X> out_x(a.r.dx, a.r.dx_stride, p - Sh::TILE), out_a(a.r.da, a.r.da_stride, p - Sh::TILE);
#pragma unroll
      for (int i = T - 1; i >= 0; --i) {
        const bool last = ends >> i & 1;
        float dx[V], da[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float g = last ? d[i][e] : d[i][e] + c[e];
          dx[e] = in[i][e] * g;
          da[e] = dx[e] * (diff[i][e] * f[i][e]);
          c[e] = f[i][e] * g;
        }
        if (i >= skip) {
          col.store(out_x.at(i, place_dx), dx);
          col.store(out_a.at(i, place_da), da);
        }
        if (a.r.dh0 && (starts >> i & 1)) col.store(a.r.dh0 + Bounds<T>::sequence(a, q + i) * a.r.D + col.at, c);
      }
    }
  }
  if constexpr (MAP) {
    if ((int)threadIdx.x < LPC) {
      store_vec<float, V>(a.part_F + (int64_t)part * a.r.D + col.at, carry.F);
      store_vec<float, V>(a.part_S + (int64_t)part * a.r.D + col.at, carry.S);
    }
    if (threadIdx.x == 0) a.part_forget[(int64_t)part * a.groups + group] = carry.forget;
  }
}

// One position of each of n sequences: a vector of columns a thread, `lanes` of
// them over a row's columns.
template <typename X, int V>
__global__ void __launch_bounds__(kScanBlock)
scan_step_kernel(RecurrenceArgs r, int lanes, int column_blocks) {
  const int rows = kScanBlock / lanes;
  const ScanColumns<V> col((int)((blockIdx.x % (unsigned)column_blocks) * lanes + threadIdx.x % lanes) * V, r.D);
  if (col.shift == V) return;
  const int64_t step = (int64_t)(gridDim.x / (unsigned)column_blocks) * rows;
  for (int64_t b = (int64_t)(blockIdx.x / (unsigned)column_blocks) * rows + threadIdx.x / lanes; b < r.n; b += step) {
    float x[V], g[V], h[V] = {};
    load_vec<X, V>(static_cast<const X*>(r.a) + b * r.a_stride + col.at, g);
    load_vec<X, V>(static_cast<const X*>(r.x) + b * r.x_stride + col.at, x);
    if (r.h0) load_vec<float, V>(r.h0 + b * r.D + col.at, h);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float f, i;
      gate_of<sizeof(X) == 4>(g[e], f, i);
      h[e] = __builtin_fmaf(f, h[e], i * x[e]);
    }
    col.store(static_cast<X*>(r.h) + b * r.h_stride + col.at, h);
    if (r.h_last) col.store(r.h_last + b * r.D + col.at, h);
  }
}

// ------------------------------------------------------------- launching
// The most parts that sequences are cut into: of blocks of the widest groups of columns.
static int64_t scan_most_parts(int32_t D) { return std::max<int64_t>(1, kScanBlocks / ceil_div(D, kScanWidest)); }

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
  const int64_t parts = scan_most_parts(D);
  r.seq = take((size_t)n * sizeof(int32_t));
  r.F = take((size_t)parts * D * sizeof(float));
  r.S = take((size_t)parts * D * sizeof(float));
  r.forget = take((size_t)std::max<int64_t>(kScanBlocks, D) * sizeof(int32_t));   // (parts x groups)
  r.state = take((size_t)std::min(B, kScanSplitBelow) * D * sizeof(float));
  r.bytes = at + 256;
  return r;
}
size_t recurrence_workspace_bytes(int64_t n, int64_t B, int32_t D) { return scan_room(n, B, D).bytes; }

template <typename X, int LPC, int V, bool GRAD>
static hipError_t scan_in(ScanArgs a, void* ws, hipStream_t stream) {
  constexpr int T = kScanT<GRAD>;
  typedef ScanShape<LPC, V, T> Sh;
  const RecurrenceArgs& r = a.r;
  const int64_t tiles = ceil_div(r.n, Sh::TILE);
  a.groups = (int32_t)ceil_div(r.D, Sh::COLUMNS);
  const ScanRoom room = scan_room(r.n, r.B, r.D);
  char* base = static_cast<char*>(ws);
  const int64_t most = std::max<int64_t>(1, kScanBlocks / a.groups);
  a.split = r.B * a.groups < kScanSplitBelow && most > r.B && tiles > 2 * r.B;
  const int64_t parts = std::min(most, tiles);
  if (a.split) {
    a.part_len = (int32_t)(ceil_div(ceil_div(r.n, parts), Sh::TILE) * Sh::TILE);
    a.part_F = reinterpret_cast<float*>(base + room.F);
    a.part_S = reinterpret_cast<float*>(base + room.S);
    a.part_forget = reinterpret_cast<int32_t*>(base + room.forget);
    if (GRAD ? r.dh_last && r.dh0 : r.h0 && r.h_last) a.state = reinterpret_cast<float*>(base + room.state);
  } else {
    a.part_len = (int32_t)ceil_div(r.n, parts);
    if (!a.seq) a.part_len = (int32_t)(ceil_div(a.part_len, a.length) * a.length);   // (no more than n)
  }
  a.parts = (int32_t)ceil_div(r.n, a.part_len);
  const dim3 grid((unsigned)((int64_t)a.parts * a.groups));
  if constexpr (GRAD) {
    if (a.split) hipLaunchKernelGGL((scan_grad_kernel<X, LPC, V, T, true>), grid, dim3(kScanBlock), 0, stream, a);
    hipLaunchKernelGGL((scan_grad_kernel<X, LPC, V, T, false>), grid, dim3(kScanBlock), 0, stream, a);
  } else {
    if (a.split) hipLaunchKernelGGL((scan_kernel<X, LPC, V, T, true>), grid, dim3(kScanBlock), 0, stream, a);
    hipLaunchKernelGGL((scan_kernel<X, LPC, V, T, false>), grid, dim3(kScanBlock), 0, stream, a);
  }
  return hipGetLastError();
}

template <typename X, int V>
static hipError_t scan_step(const RecurrenceArgs& r, hipStream_t stream) {
  const int64_t vecs = ceil_div(r.D, V);
  int lanes = 1;
  while (lanes < kScanBlock && lanes < vecs) lanes *= 2;
  const int64_t columns = ceil_div(vecs, lanes), rows = kScanBlock / lanes;
  const int64_t blocks = std::min(ceil_div(r.n, rows), std::max<int64_t>(1, (int64_t(1) << 20) / columns));
  hipLaunchKernelGGL((scan_step_kernel<X, V>), dim3((unsigned)(blocks * columns)), dim3(kScanBlock), 0, stream, r, lanes,
                     (int)columns);
  return hipGetLastError();
}

template <typename X, bool GRAD>
static hipError_t scan_as(const ScanArgs& a, void* ws, hipStream_t stream) {
  constexpr int V = kScanV;
  const int32_t D = a.r.D;
  if (!GRAD && !a.seq && a.length == 1) return D < V ? scan_step<X, 1>(a.r, stream) : scan_step<X, V>(a.r, stream);
  if (D < V) return scan_in<X, 4, 1, GRAD>(a, ws, stream);
  if (D <= 4 * V) return scan_in<X, 4, V, GRAD>(a, ws, stream);
  if (D <= 8 * V) return scan_in<X, 8, V, GRAD>(a, ws, stream);
  // fewer columns to a block where the sequences are then enough blocks, and are too few for what memory takes at once
  const int64_t blocks = a.r.B * ceil_div(D, kScanWidest);
  const bool few = blocks * (int64_t)sizeof(X) < kScanBlocks * 2 && 2 * blocks >= kScanSplitBelow;
  if (D <= 16 * V || few) return scan_in<X, 16, V, GRAD>(a, ws, stream);
  return scan_in<X, kScanLanes, V, GRAD>(a, ws, stream);
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
    const int64_t blocks = std::min<int64_t>(ceil_div(work, kScanBlock), 1024);
    hipLaunchKernelGGL(scan_map_kernel, dim3((unsigned)blocks), dim3(kScanBlock), 0, stream, m);
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
