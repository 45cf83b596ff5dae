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
// Positions are cut into parts, one for a block and group of columns.  Equal
// lengths: of whole sequences where there are enough of them.  Few long ones, and
// packed ones of any lengths, are cut where the parts come out equal, and a first
// launch maps what a part hands on to the next: the positions from its last
// sequence's beginning on (nothing where that ends with the part).  A block of the
// second launch joins the maps of those parts that the sequence passes before.
//
// Bound by bytes: 32 sequences of 1024 positions of 2048 columns bf16 94 to 98 us (403 MB,
// 4.2 TB/s where a large copy has 5.2), their like of 1024 columns f32 75; the
// gradient over 16 of 2048 of 2048 bf16 172 us (805 MB, 4.7 TB/s).  Cut sequences
// are read twice in part: the gradient over one of 100,003 positions of 511
// columns f32 336 us, of which the maps are 74.
#include <algorithm>

#include "elements.hpp"
#include "gba_device.hpp"
#include "gba_internal.hpp"

namespace gba {

constexpr int kScanBlock = 256;
constexpr int kScanWaves = kScanBlock / kWave;
// Columns of a lane, and most lanes over the columns of a block: rows by 256 or 512
// bytes (one sequence of 100,003 x 511 f32, the gradient: by 128 bytes 525 us, 256 449,
// 512 385).  With two columns of a lane twice as many loads: 32 x 1024 x 2048 bf16
// 110 us -> 126; with eight (16 bytes of bf16) 112.
constexpr int kScanV = 4;
constexpr int kScanLanes = 32;
constexpr int kScanWidest = kScanLanes * kScanV;
// Waves of a SIMD that the registers are for: with three or four of them and tiles of
// half as many positions, or with spilled registers, the same 125 to 140 us.
constexpr int kScanSimd = 2;
// Blocks of a round, a wave of each on every SIMD, that parts are made for: histories
// of 4096 users of 64 columns, cut between sequences, 48 us, with twice as many parts 52,
// four times 59.
constexpr int64_t kScanBlocks = 256 * kScanSimd;
// Sequences of equal length are cut below as many blocks of whole ones: the maps read
// two arrays again, of three or (the gradient's) six.
constexpr int64_t kScanSplitBelow = 192;

__host__ __device__ static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

// ---------------------------------------------------------------- the gate
// f = sigmoid(a) and i = 1 - f, each within a few u of itself (0 below the normal
// numbers), or (not FINE: 16-bit types, whose values carry 2^-9 or 2^-12 anyway)
// |a| u more, also in the states of 32 bits.
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

// ------------------------------------------------------------ the positions
struct ScanArgs {
  RecurrenceArgs r;
  int32_t* seq;            // packed: the sequence of each position (-1 behind the last); null: equal lengths
  int32_t length;          // ... of this many positions
  int32_t groups;          // of columns
  int32_t parts;           // of the positions
  int32_t part_len;        // positions of a part
  struct ScanPart* part;   // [parts] (null: parts of whole sequences)
  float* part_F;           // [parts][D] the parts' maps
  float* part_S;
  float* state;            // [parts][D] the state (or gradient) that a sequence begins (ends) with in a part and leaves
                           // it, where its own place is written over by another block; may be null
};

// What the first launch leaves of a part.
struct ScanPart {
  int32_t end;             // where its positions end
  int32_t from;            // the part in which the sequence begins that it is entered in the middle of (GRAD: ends), or -1
  int32_t on;              // the sequence that goes on behind it (GRAD: in front of it), or -1
  int32_t unused;
};

// Where sequence b begins and ends.
__device__ __forceinline__ int64_t seq_begin(const ScanArgs& a, int64_t b) {
  return a.seq ? a.r.offsets[b] : b * a.length;
}
__device__ __forceinline__ int64_t seq_end(const ScanArgs& a, int64_t b) {
  return a.seq ? a.r.offsets[b + 1] : (b + 1) * a.length;
}
// For each of two positions the last b of 0 .. B - 1 with offsets[b] <= p, or 0: the wave reads 64 of them at once.
__device__ __forceinline__ void wave_find(const int64_t* offsets, int64_t B, int64_t p, int64_t q, int64_t& b, int64_t& c) {
  b = c = 0;
  for (int64_t width = B; width > 1;) {
    const int64_t step = (width + kWave - 1) / kWave, i = b + lane_id() * step, j = c + lane_id() * step;
    const bool in = lane_id() * step < width;
    const int64_t x = in && i < B ? offsets[i] : INT64_MAX, y = in && j < B ? offsets[j] : INT64_MAX;
    const uint64_t up_to_p = __ballot(x <= p) | 1u, up_to_q = __ballot(y <= q) | 1u;
    b += (63 - __clzll(up_to_p)) * step;
    c += (63 - __clzll(up_to_q)) * step;
    width = step;
  }
}

// Where a block is in the order of parts and groups: blocks go to the eight dies
// in turn, and neighbours, which read the same rows, come to one die (the gradient
// of 100,003 x 511 f32 449 us -> 437, of 16 x 2048 x 2048 bf16 182 -> 173).
__device__ __forceinline__ unsigned block_place(unsigned n) {
  constexpr unsigned kDies = 8;
  const unsigned each = n / kDies, more = n % kDies, die = blockIdx.x % kDies;
  return die * each + (die < more ? die : more) + blockIdx.x / kDies;
}
// Packed sequences: the sequence of each of a part's positions.
__device__ __forceinline__ void write_sequences(const ScanArgs& a, int part, int group) {
  const int64_t* offsets = a.r.offsets;
  const int64_t p0 = (int64_t)part * a.part_len, p1 = p0 + a.part_len < a.r.n ? p0 + a.part_len : a.r.n;
  int64_t first, last;
  wave_find(offsets, a.r.B, p0, p1 - 1, first, last);
  const int64_t to = p0 + (p1 - p0) * (group + 1) / a.groups;   // the groups' blocks share the part
  for (int64_t p = p0 + (p1 - p0) * group / a.groups + threadIdx.x; p < to; p += kScanBlock) {
    int64_t lo = first, hi = last + 1;
    while (hi - lo > 1) {
      const int64_t mid = (lo + hi) >> 1;
      if (offsets[mid] <= p) lo = mid;
      else hi = mid;
    }
    a.seq[p] = offsets[lo] <= p && p < offsets[lo + 1] ? (int32_t)lo : -1;
  }
}
// The checks of the offsets, and what an empty sequence hands on: its state, or
// its state's gradient: block `block` of `blocks`, a wave every (waves)-th
// sequence, 64 at a time.
template <bool GRAD>
__device__ __forceinline__ void check_sequences(const ScanArgs& a, unsigned block, unsigned blocks, int32_t* err) {
  const int64_t* offsets = a.r.offsets;
  const int64_t B = a.r.B, D = a.r.D, waves = (int64_t)blocks * kScanWaves;
  float* to = GRAD ? a.r.dh0 : a.r.h_last;
  const float* from = GRAD ? a.r.dh_last : a.r.h0;
  if (to == from) to = nullptr;
  for (int64_t b0 = (int64_t)block * kScanWaves + threadIdx.x / kWave; b0 < B; b0 += waves * kWave) {
    const int64_t b = b0 + lane_id() * waves;
    const int64_t begin = b < B ? offsets[b] : 0, end = b < B ? offsets[b + 1] : 1;
    if (begin > end || (b == 0 && begin != 0) || (b < B && end > a.r.n)) raise_error(err, GBA_DERR_OFFSETS);
    if (!to) continue;
    for (uint64_t empty = __ballot(begin >= end); empty; empty &= empty - 1) {
      const int64_t row = (b0 + (__ffsll((unsigned long long)empty) - 1) * waves) * D;
#pragma unroll 4
      for (int64_t c = lane_id() * 4; c < D; c += kWave * 4) {
        float v[4] = {};
        if (from) load_part<float, 4>(from + row + c, (int)(D - c), v);
        store_part<float, 4>(to + row + c, (int)(D - c), v);
      }
    }
  }
}

// ------------------------------------------------------------ the kernels
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

// Positions of a lane: what the registers hold beside the next tile (4 forward:
// 32 x 1024 x 2048 bf16 100 us -> 125; 2 backward: 16 x 2048 x 2048 bf16 185 -> 199, 5 203).
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
// (JOIN: how many waves' maps are read at a time)
template <int LPC, int V, bool MAP, int JOIN = kScanWaves>
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
  Affine<V> tile;
  if constexpr (MAP) tile.clear();
  __syncthreads();
#pragma unroll JOIN
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
      b.after(tile);
      tile = b;
    } else {
      b.apply(carry.S);
    }
  }
  if constexpr (MAP) carry.after(tile);
  buffer ^= 1;
  if constexpr (!MAP)
    if (lane >= LPC) x.apply(in);
}

// The state that a part is entered with (in carry.S): the maps of `count` parts
// from `first` on (back to front with BACK), each slot a share of them.
template <int LPC, int V, bool BACK>
__device__ __forceinline__ void enter_part(const ScanArgs& a, int first, int count, int col, Affine<V>& carry, int& buffer,
                                           ScanShared<LPC, V>& s) {
  constexpr int SLOTS = kScanBlock / LPC;
  const int slot = threadIdx.x / LPC;
  const int lo = (int)((int64_t)count * slot / SLOTS), hi = (int)((int64_t)count * (slot + 1) / SLOTS);
  Affine<V> m;
  m.clear();
#pragma unroll 4
  for (int k = lo; k < hi; ++k) {
    const int64_t j = BACK ? first - k : first + k;
    Affine<V> b;
    load_vec<float, V>(a.part_F + j * a.r.D + col, b.F);
    load_vec<float, V>(a.part_S + j * a.r.D + col, b.S);
    b.forget = false;
    b.after(m);
    m = b;
  }
  float unused[V];
  scan_join<LPC, V, false>(m, carry, unused, buffer, s);
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
// registers, twice as many as the tile itself takes: the gradient of f32 spilled
// 276 bytes of a lane).
template <typename X>
__device__ __forceinline__ uint64_t lane_place(int64_t stride, int64_t row, int col) {
  return (uint64_t)(row * stride + col) * sizeof(X);
}
__device__ __forceinline__ void keep_place(uint64_t& place) { asm volatile("" : "+v"(place)); }

// A matrix's rows from a uniform one on.  Read and (ScanColumns) written past the
// caches, each being touched once: 32 x 1024 x 2048 bf16 109 us -> 103, the gradient of
// 16 x 2048 x 2048 186 -> 177, of 100,003 x 511 f32 382 -> 353.
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
  template <int V, bool PAST = true>
  __device__ __forceinline__ typename VecOf<X, V>::type load(int i, uint64_t place) const {
    typedef typename VecOf<X, V>::type vec;
    const vec* p = reinterpret_cast<const vec*>(at(i, place));
    return PAST ? __builtin_nontemporal_load(p) : *p;
  }
};

// The map of what a part hands on.  Forward: of its positions from the last
// sequence's beginning on; GRAD: back from the first sequence's end.
template <typename X, int LPC, int V, bool GRAD>
__device__ __forceinline__ void map_part(const ScanArgs& a, int part, int group, ScanShared<LPC, V>& s) {
  constexpr int T = kScanT<false>;
  typedef ScanShape<LPC, V, T> Sh;
  typedef typename VecOf<X, V>::type vec;
  const int64_t p0 = (int64_t)part * a.part_len;
  int64_t p1 = p0 + a.part_len < a.r.n ? p0 + a.part_len : a.r.n;
  int64_t used = a.r.n, first, last;
  if (a.seq) {
    used = a.r.offsets[a.r.B];
    wave_find(a.r.offsets, a.r.B, p0, p1 - 1, first, last);
  } else {
    first = (uint32_t)p0 / (uint32_t)a.length;
    last = (uint32_t)(p1 - 1) / (uint32_t)a.length;
  }
  // (of the first and of the last position: those behind the last sequence are in none)
  const int64_t begin0 = seq_begin(a, first), end0 = seq_end(a, first), begin1 = seq_begin(a, last), end1 = seq_end(a, last);
  const bool before = begin0 < p0 && end0 > p0, behind = begin1 < p1 && end1 > p1;
  if (group == 0 && threadIdx.x == 0) {
    ScanPart o;
    o.end = (int32_t)(used < 0 ? 0 : used < p1 ? used : p1);
    const int64_t there = GRAD ? (end1 < a.r.n ? end1 : a.r.n) - 1 : (begin0 < 0 ? 0 : begin0);
    o.from = (GRAD ? behind : before) ? (int32_t)((uint32_t)there / (uint32_t)a.part_len) : -1;
    o.on = (GRAD ? before : behind) ? (int32_t)(GRAD ? first : last) : -1;
    o.unused = 0;
    a.part[part] = o;
  }
  // the sequence that goes on, and its positions here
  if (GRAD ? !before : !behind) return;
  const int64_t b = GRAD ? first : last;
  const bool forget = GRAD ? end0 <= p1 : begin1 >= p0;   // it begins (ends) here
  const int64_t q0 = __builtin_amdgcn_readfirstlane((int)(!GRAD && forget ? begin1 : p0));
  const int64_t q1 = __builtin_amdgcn_readfirstlane((int)(GRAD && forget ? end0 : p1));

  const int slot = threadIdx.x / LPC;
  const ScanColumns<V> col(group * Sh::COLUMNS + (int)(threadIdx.x % LPC) * V, a.r.D);
  const int place = GRAD ? (Sh::SLOTS - 1 - slot) * T : slot * T;   // of the slot in a tile
  const void* const in = GRAD ? a.r.dh : a.r.x;
  const int64_t in_stride = GRAD ? a.r.dh_stride : a.r.x_stride;
  uint64_t place_a = lane_place<X>(a.r.a_stride, place, col.at), place_x = lane_place<X>(in_stride, place, col.at);
  float h0[V] = {};
  if (forget) {
    const float* from = GRAD ? a.r.dh_last : a.r.h0;
    if (from) load_vec<float, V>(from + b * a.r.D + col.at, h0);
    if (a.state && slot == 0) col.store(a.state + (int64_t)part * a.r.D + col.at, h0);
  }
  vec x[T] = {}, g[T] = {};
  auto load = [&](int64_t t) {   // the tile that begins at t
    keep_place(place_a);
    keep_place(place_x);
    const RowsFrom<X> rows_a(a.r.a, a.r.a_stride, t), rows_x(in, in_stride, t);
    const int64_t q = t + place;
    if (t >= q0 && t + Sh::TILE <= q1) {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        g[i] = rows_a.template load<V, false>(i, place_a);
        x[i] = rows_x.template load<V, false>(i, place_x);
      }
    } else {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (q + i < q0 || q + i >= q1) continue;
        g[i] = rows_a.template load<V, false>(i, place_a);
        x[i] = rows_x.template load<V, false>(i, place_x);
      }
    }
  };
  int buffer = 0;
  Affine<V> carry;
  carry.clear();
  const int64_t tiles = (q1 - q0 + Sh::TILE - 1) / Sh::TILE;
  // the tiles the other way round than the second launch, and through the caches, where it finds the last ones (the gradient
  // over 100,003 x 511 f32 357 us -> 336, over 2 x 50,000 x 512 bf16 178 -> 172, forward 126 -> 120; histories the same)
  auto tile = [&](int64_t k) { return GRAD ? q1 - (tiles - k) * Sh::TILE : q0 + (tiles - 1 - k) * Sh::TILE; };
  load(tile(0));
  for (int64_t k = 0; k < tiles; ++k) {
    const int64_t t = tile(k), q = t + place;
    float f[T][V], v[T][V];
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        gate_of<sizeof(X) == 4>((float)g[i][e], f[i][e], v[i][e]);
        v[i][e] = GRAD ? (float)x[i][e] : v[i][e] * (float)x[i][e];
      }
    if (k + 1 < tiles) load(tile(k + 1));
    if (t < q0 || t + Sh::TILE > q1) {   // beyond the positions: steps that do nothing
#pragma unroll
      for (int i = 0; i < T; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const bool here = q + i >= q0 && q + i < q1;
          f[i][e] = here ? f[i][e] : 1.0f;
          v[i][e] = here ? v[i][e] : 0.0f;
        }
    }
    Affine<V> m;
    m.forget = false;
    if constexpr (GRAD) {
      const bool last = k == tiles - 1 && slot == 0 && forget;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        m.S[e] = f[T - 1][e] * (last ? v[T - 1][e] + h0[e] : v[T - 1][e]);
        m.F[e] = f[T - 1][e];
      }
#pragma unroll
      for (int i = T - 2; i >= 0; --i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          m.S[e] = f[i][e] * (v[i][e] + m.S[e]);
          m.F[e] *= f[i][e];
        }
    } else {
      const bool first = k == tiles - 1 && slot == 0 && forget;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        m.S[e] = first ? __builtin_fmaf(f[0][e], h0[e], v[0][e]) : v[0][e];
        m.F[e] = f[0][e];
      }
#pragma unroll
      for (int i = 1; i < T; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          m.S[e] = __builtin_fmaf(f[i][e], m.S[e], v[i][e]);
          m.F[e] *= f[i][e];
        }
    }
    float unused[V];
    scan_join<LPC, V, true>(m, carry, unused, buffer, s);
  }
  // (where it begins here F is multiplied by the 0 that it is entered with)
  if (slot == 0 && col.shift < V) {
    store_vec<float, V>(a.part_F + (int64_t)part * a.r.D + col.at, carry.F);
    store_vec<float, V>(a.part_S + (int64_t)part * a.r.D + col.at, carry.S);
  }
}
template <typename X, int LPC, int V, bool GRAD>
__global__ void __launch_bounds__(kScanBlock, kScanSimd)
scan_part_kernel(ScanArgs a, int32_t* err) {
  __shared__ ScanShared<LPC, V> s;
  const unsigned blocks = (unsigned)a.parts * (unsigned)a.groups, groups = (unsigned)a.groups;
  if (blockIdx.x < blocks) {
    const unsigned block = block_place(blocks);
    map_part<X, LPC, V, GRAD>(a, (int)(block / groups), (int)(block % groups), s);
  } else {   // packed: beside the maps
    const unsigned block = blockIdx.x - blocks;
    if (block < blocks) write_sequences(a, (int)(block / groups), (int)(block % groups));
    check_sequences<GRAD>(a, block, gridDim.x - blocks, err);
  }
}

template <typename X, int LPC, int V, int T>
__global__ void __launch_bounds__(kScanBlock, kScanSimd)
scan_kernel(ScanArgs a) {
  typedef ScanShape<LPC, V, T> Sh;
  typedef typename VecOf<X, V>::type vec;
  __shared__ ScanShared<LPC, V> s;
  const unsigned block = block_place(gridDim.x);
  const int group = (int)(block % (unsigned)a.groups), part = (int)(block / (unsigned)a.groups);
  const int slot = threadIdx.x / LPC;
  const ScanColumns<V> col(group * Sh::COLUMNS + (int)(threadIdx.x % LPC) * V, a.r.D);
  const int64_t p0 = (int64_t)part * a.part_len;
  int64_t p1 = p0 + a.part_len < a.r.n ? p0 + a.part_len : a.r.n;
  int from = -1, on = -1;
  if (a.part) {   // (the same in every lane, also to the compiler)
    p1 = __builtin_amdgcn_readfirstlane(a.part[part].end);
    from = __builtin_amdgcn_readfirstlane(a.part[part].from);
    on = __builtin_amdgcn_readfirstlane(a.part[part].on);
  }
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
  if (p0 >= p1) return;
  load(p0);
  if (from >= 0) enter_part<LPC, V, false>(a, from, part - from, col.at, carry, buffer, s);
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
    if (starts && a.r.h0) {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (!(starts >> i & 1)) continue;
        const int64_t b = Bounds<T>::sequence(a, q + i);
        const float* row = a.state && b == on ? a.state + (int64_t)part * a.r.D : a.r.h0 + b * a.r.D;
        float h0[V];
        load_vec<float, V>(row + col.at, h0);
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
    scan_join<LPC, V, false>(m, carry, h, buffer, s);
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

// The gradient: positions from the end; slot 0 takes a tile's last ones.  The
// state that runs through is f_t g_t, what a position hands to the one before it.
template <typename X, int LPC, int V, int T>
__global__ void __launch_bounds__(kScanBlock, kScanSimd)
scan_grad_kernel(ScanArgs a) {
  typedef ScanShape<LPC, V, T> Sh;
  typedef typename VecOf<X, V>::type vec;
  __shared__ ScanShared<LPC, V> s;
  const unsigned block = block_place(gridDim.x);
  const int group = (int)(block % (unsigned)a.groups), part = (int)(block / (unsigned)a.groups);
  const int slot = threadIdx.x / LPC;
  const ScanColumns<V> col(group * Sh::COLUMNS + (int)(threadIdx.x % LPC) * V, a.r.D);
  const int64_t p0 = (int64_t)part * a.part_len;
  int64_t p1 = p0 + a.part_len < a.r.n ? p0 + a.part_len : a.r.n;
  int from = -1, on = -1;
  if (a.part) {   // (the same in every lane, also to the compiler)
    p1 = __builtin_amdgcn_readfirstlane(a.part[part].end);
    from = __builtin_amdgcn_readfirstlane(a.part[part].from);
    on = __builtin_amdgcn_readfirstlane(a.part[part].on);
  }
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
        x[i] = rows_x.template load<V>(i, place_x);
        before[i] = rows_h.template load<V>(i, place_h);
      }
    } else {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (q + i < p0) continue;
        gate[i] = rows_a.template load<V>(i, place_a);
        dh[i] = rows_d.template load<V>(i, place_d);
        x[i] = rows_x.template load<V>(i, place_x);
        if (q + i > 0) before[i] = rows_h.template load<V>(i, place_h);
      }
    }
    at.load(a, q);
  };
  if (p0 >= p1) return;
  load(p1);
  if (from >= 0) enter_part<LPC, V, true>(a, from, from - part, col.at, carry, buffer, s);
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
        diff[i][e] = (float)before[i][e] - (float)x[i][e];
      }
    // (what slots in front of the part compute goes nowhere)
    at.find(a, q, skip, T);
    const uint32_t starts = at.starts, ends = at.ends;
    if (starts) {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (!(starts >> i & 1)) continue;
        float h0[V] = {};
        if (a.r.h0) load_vec<float, V>(a.r.h0 + Bounds<T>::sequence(a, q + i) * a.r.D + col.at, h0);
#pragma unroll
        for (int e = 0; e < V; ++e) diff[i][e] = h0[e] - (float)x[i][e];
      }
    }
    if (ends && a.r.dh_last) {
#pragma unroll
      for (int i = 0; i < T; ++i) {
        if (!(ends >> i & 1)) continue;
        const int64_t b = Bounds<T>::sequence(a, q + i);
        const float* row = a.state && b == on ? a.state + (int64_t)part * a.r.D : a.r.dh_last + b * a.r.D;
        float g[V];
        load_vec<float, V>(row + col.at, g);
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
    // (32 bits: four waves' maps at a time would not fit the registers, 32 x 1024 positions of 1024 157 us to 140)
    scan_join<LPC, V, false, sizeof(X) == 4 ? 2 : kScanWaves>(m, carry, c, buffer, s);
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
// The most parts that are made: of blocks of the widest groups of columns.
static int64_t scan_most_parts(int32_t D) { return std::max<int64_t>(1, kScanBlocks / ceil_div(D, kScanWidest)); }

// The sequence of each position, and the parts' maps and states.
struct ScanRoom {
  size_t seq, part, F, S, state, bytes;
};
static ScanRoom scan_room(int64_t n, int32_t D) {
  ScanRoom r;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align_up(bytes);
    return here;
  };
  const size_t rows = (size_t)scan_most_parts(D) * D * sizeof(float);
  r.seq = take((size_t)n * sizeof(int32_t));
  r.part = take((size_t)scan_most_parts(D) * sizeof(ScanPart));
  r.F = take(rows);
  r.S = take(rows);
  r.state = take(rows);
  r.bytes = at + 256;
  return r;
}
size_t recurrence_workspace_bytes(int64_t n, int64_t, int32_t D) { return scan_room(n, D).bytes; }

template <typename X, int LPC, int V, bool GRAD>
static hipError_t scan_in(ScanArgs a, void* ws, int32_t* err, hipStream_t stream) {
  constexpr int T = kScanT<GRAD>;
  typedef ScanShape<LPC, V, T> Sh;
  const RecurrenceArgs& r = a.r;
  const int64_t tiles = ceil_div(r.n, Sh::TILE);
  a.groups = (int32_t)ceil_div(r.D, Sh::COLUMNS);
  const int64_t parts = std::max<int64_t>(1, std::min(std::max<int64_t>(1, kScanBlocks / a.groups), tiles));
  a.part_len = (int32_t)std::max<int64_t>(1, ceil_div(r.n, parts));
  const bool split = a.seq || (r.B * a.groups < kScanSplitBelow && tiles > 2 * r.B);
  if (split) {
    const ScanRoom room = scan_room(r.n, r.D);
    char* base = static_cast<char*>(ws);
    a.part_len = (int32_t)std::min<int64_t>(ceil_div(a.part_len, Sh::TILE) * Sh::TILE, INT32_MAX);
    a.part = reinterpret_cast<ScanPart*>(base + room.part);
    a.part_F = reinterpret_cast<float*>(base + room.F);
    a.part_S = reinterpret_cast<float*>(base + room.S);
    if (GRAD ? r.dh_last && r.dh0 : r.h0 && r.h_last) a.state = reinterpret_cast<float*>(base + room.state);
  } else {
    // (no more than n; one sequence more than blocks of one round take makes two of each block: 32 x 1024 x 2048 bf16 98 us,
    // 33 164, 64 176)
    a.part_len = (int32_t)(ceil_div(a.part_len, a.length) * a.length);
  }
  a.parts = (int32_t)ceil_div(r.n, a.part_len);
  const int64_t blocks = (int64_t)a.parts * a.groups;
  if (split) {
    const int64_t beside = a.seq ? std::max(blocks, std::min<int64_t>(ceil_div(r.B, kScanWaves), 1024)) : 0;
    hipLaunchKernelGGL((scan_part_kernel<X, LPC, V, GRAD>), dim3((unsigned)(blocks + beside)), dim3(kScanBlock), 0, stream,
                       a, err);
  }
  if (r.n == 0) return hipGetLastError();
  const dim3 grid((unsigned)blocks);
  if constexpr (GRAD) hipLaunchKernelGGL((scan_grad_kernel<X, LPC, V, T>), grid, dim3(kScanBlock), 0, stream, a);
  else hipLaunchKernelGGL((scan_kernel<X, LPC, V, T>), grid, dim3(kScanBlock), 0, stream, a);
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
static hipError_t scan_as(const ScanArgs& a, void* ws, int32_t* err, hipStream_t stream) {
  constexpr int V = kScanV;
  const int32_t D = a.r.D;
  if (!GRAD && !a.seq && a.length == 1) return D < V ? scan_step<X, 1>(a.r, stream) : scan_step<X, V>(a.r, stream);
  if (D < V) return scan_in<X, 4, 1, GRAD>(a, ws, err, stream);
  if (D <= 4 * V) return scan_in<X, 4, V, GRAD>(a, ws, err, stream);
  if (D <= 8 * V) return scan_in<X, 8, V, GRAD>(a, ws, err, stream);
  // 64 columns to a block, not 128, where these are too few blocks for what memory takes at once (the gradient of
  // 16 x 2048 x 2048 bf16 225 us -> 175; but 256 blocks of f32 are enough: 32 x 1024 x 1024 75, with 64 columns 86)
  const int64_t blocks = a.r.B * ceil_div(D, kScanWidest);
  const bool few = !a.seq && blocks * (int64_t)sizeof(X) < kScanBlocks * 2 && 2 * blocks >= kScanSplitBelow;
  if (D <= 16 * V || few) return scan_in<X, 16, V, GRAD>(a, ws, err, stream);
  return scan_in<X, kScanLanes, V, GRAD>(a, ws, err, stream);
}

// Sequences of no positions at all: each hands on its state, or its state's gradient.
__global__ void __launch_bounds__(kScanBlock)
scan_empty_kernel(const float* __restrict__ from, float* __restrict__ to, int64_t count) {
  const int64_t step = (int64_t)gridDim.x * kScanBlock;
  for (int64_t i = (int64_t)blockIdx.x * kScanBlock + threadIdx.x; i < count; i += step) to[i] = from ? from[i] : 0.0f;
}
static hipError_t scan_empty(const float* from, float* to, int64_t count, hipStream_t stream) {
  if (!to || to == from) return hipSuccess;
  const int64_t blocks = std::min(ceil_div(count, kScanBlock), int64_t(1) << 20);
  hipLaunchKernelGGL(scan_empty_kernel, dim3((unsigned)blocks), dim3(kScanBlock), 0, stream, from, to, count);
  return hipGetLastError();
}

template <bool GRAD>
static hipError_t launch_scan(const RecurrenceArgs& r, void* ws, int32_t* err, hipStream_t stream) {
  if (r.n == 0 && !r.offsets)
    return GRAD ? scan_empty(r.dh_last, r.dh0, r.B * r.D, stream) : scan_empty(r.h0, r.h_last, r.B * r.D, stream);
  ScanArgs a{};
  a.r = r;
  if (r.offsets) a.seq = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + scan_room(r.n, r.D).seq);
  else a.length = (int32_t)(r.n / r.B);
  if (r.type == GBA_F32) return scan_as<float, GRAD>(a, ws, err, stream);
  if (r.type == GBA_BF16) return scan_as<bf16_t, GRAD>(a, ws, err, stream);
  return scan_as<f16_t, GRAD>(a, ws, err, stream);
}

hipError_t launch_recurrence(const RecurrenceArgs& r, void* ws, int32_t* err, hipStream_t stream) {
  return launch_scan<false>(r, ws, err, stream);
}
hipError_t launch_recurrence_grad(const RecurrenceArgs& r, void* ws, int32_t* err, hipStream_t stream) {
  return launch_scan<true>(r, ws, err, stream);
}

}  // namespace gba
