// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// The gradient: the tokens are sorted by ID (the push path's stable sort), and
// the sorted list is cut into blocks of positions whatever the IDs, so that a
// frequent ID's tokens are shared among many lane groups.  A lane group adds
// up the gradient rows of its positions; an ID that begins and ends inside the
// group goes straight to the output, what crosses a group's edge is joined
// within the block by the group where the ID begins, and what crosses a
// block's edge by a second launch, through 32-bit partial rows.  Every sum has one order, so the
// same inputs give the same bits, and no atomic is used.
#include <algorithm>

#include "elements.hpp"
#include "gba_device.hpp"
#include "gba_internal.hpp"
#include "run_heads.hpp"

namespace gba {

constexpr int kEmbBlock = 256;
constexpr int kEmbWaves = kEmbBlock / kWave;
constexpr int64_t kMaxGrid = 1 << 20;
constexpr int64_t kMostBlocks = (int64_t(1) << 24) - 1;   // of a launch: 2^32 threads

__host__ __device__ static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

// Lanes that share a row slice of V elements each: a power of two, up to a wave.
static int lanes_for(int32_t D, int V) {
  int l = 1;
  while (l < kWave && l * V < D) l <<= 1;
  return l;
}

// Where a thread's V columns of a row lie.  The last vector of a row is moved
// back to end with it: its first `shift` elements are another thread's, which
// computes and stores the same values.
template <int V>
struct Columns {
  int c, shift, D;
  bool on;       // the thread has columns
  bool tiny;     // rows narrower than a vector: element by element
  __device__ __forceinline__ Columns(int first, int width) : D(width) {
    on = first < width;
    tiny = width < V;
    c = tiny ? 0 : (first + V > width ? width - V : first);
    shift = tiny ? 0 : first - c;
  }
};

// ---------------------------------------------------------------- lookup
// 2^shift threads a row and step of V columns each: 16 bytes of the output, so
// that a wave's stores leave no gaps.  Bound by the bytes of the output and of
// the distinct rows: 32,768 x 4096 bf16 57 us, 344 MB at 6.0 TB/s; 8 x 2048, one
// wave's two dependent loads, 2.6.  (Two or four rows a thread at a time: 72 us
// where one row takes 64.)  A large output is stored past the caches, PAST:
// what reads it next then finds more of its other inputs there, and the call
// itself takes 64 us instead of 81.  A small one is better left in them:
// followed by a layer norm, 8192 x 4096 bf16 take 57 us and 61 past the
// caches, 16,384 x 4096 115 and 111.  Narrow rows through a pull's inverse map,
// 256,000 of 32 f32 from 72,000: 10.8 us and 7.5 into bf16, all of it the kernel's
// (a floor of 6.2 and 3.9); 26,624 of 64 into bf16 5.9, the kernel 3.1.
constexpr int64_t kPastCaches = int64_t(96) << 20;   // bytes
template <typename T, typename O, bool PAST>
__global__ void __launch_bounds__(kEmbBlock)
lookup_kernel(LookupArgs a, int shift) {
  constexpr int V = kVec<O>;
  const int per = 1 << shift, t = threadIdx.x & (per - 1);
  const int64_t r = (int64_t)blockIdx.x * (kEmbBlock >> shift) + (threadIdx.x >> shift);
  if (r >= a.n) return;
  const int64_t id = a.id_bytes == 8 ? static_cast<const int64_t*>(a.ids)[r] : static_cast<const int32_t*>(a.ids)[r];
  const bool ok = (uint64_t)id < (uint64_t)a.R;
  if (!ok && t == 0) raise_error(a.err, GBA_DERR_ID_RANGE);
  const T* row = static_cast<const T*>(a.table) + (ok ? id : 0) * a.table_stride;
  O* out = static_cast<O*>(a.out) + r * a.out_stride;
  for (int first = t * V; first < a.D; first += per * V) {
    const Columns<V> at(first, a.D);
    const int count = at.tiny ? at.D : V;
    float v[V];
    load_part<T, V>(row + at.c, count, v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = ok ? v[e] * a.scale : 0.0f;
    store_part<O, V, PAST>(out + at.c, count, v);
  }
}

template <typename T, typename O>
static hipError_t lookup_as(LookupArgs a, hipStream_t stream) {
  int shift = 0;
  while ((1 << shift) < kEmbBlock && (kVec<O> << shift) < a.D) ++shift;
  const bool past = a.n * a.D * (int64_t)sizeof(O) >= kPastCaches;
  // (wide rows of more than 2^24 tokens are more blocks than a launch takes)
  const int64_t most = kMostBlocks * (kEmbBlock >> shift), n = a.n;
  for (int64_t at = 0; at < n; at += most) {
    a.n = std::min(most, n - at);
    const dim3 grid((unsigned)ceil_div(a.n, kEmbBlock >> shift)), block(kEmbBlock);
    if (past) hipLaunchKernelGGL((lookup_kernel<T, O, true>), grid, block, 0, stream, a, shift);
    else hipLaunchKernelGGL((lookup_kernel<T, O, false>), grid, block, 0, stream, a, shift);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.ids = static_cast<const char*>(a.ids) + most * a.id_bytes;
    a.out = static_cast<O*>(a.out) + most * a.out_stride;
  }
  return hipSuccess;
}
template <typename T>
static hipError_t lookup_from(const LookupArgs& a, hipStream_t stream) {
  if (a.out_type == GBA_F32) return lookup_as<T, float>(a, stream);
  if (a.out_type == GBA_BF16) return lookup_as<T, bf16_t>(a, stream);
  return lookup_as<T, f16_t>(a, stream);
}

hipError_t launch_embedding_lookup(const LookupArgs& a, hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  if (a.table_type == GBA_F32) return lookup_from<float>(a, stream);
  if (a.table_type == GBA_BF16) return lookup_from<bf16_t>(a, stream);
  return lookup_from<f16_t>(a, stream);
}

// -------------------------------------------------------------- gradient
constexpr int kRows = 4;             // gradient rows of a batch: twice as many loads in flight per lane group
constexpr int kMaxPos = 1024;        // most positions of a block

struct GradScratch {
  RunHeads heads;          // one row per distinct ID: where the blocks' numbering begins
  float* pieces;           // [blocks][2][D]: what the block's first ID adds to an ID of an earlier block, and the
                           // block's part of an ID that begins in it and goes on in the next
  uint32_t* tail_run;      // [blocks] the row of that second ID (one row per distinct ID)
  int span;                // positions of a lane group
  int pos;                 // ... and of a block: a power of two, at most kMaxPos
  int slices;              // column slices
  unsigned blocks;         // blocks of positions
};

// The first position whose key is not below `key` in keys[0, n): 64 probes a
// step, by one wave.
__device__ __forceinline__ int64_t wave_lower_bound(const uint32_t* __restrict__ keys, int64_t n, uint64_t key) {
  int64_t lo = 0, len = n;   // the answer is in [lo, lo + len]
  while (len > 0) {
    const int64_t step = (len + kWave - 1) / kWave;
    const int64_t at = lo + (int64_t)lane_id() * step;
    const bool below = at < lo + len && keys[at] < key;
    const int m = __popcll(__ballot(below));   // the probes ascend: a prefix of the lanes
    if (m == 0) return lo;
    const int64_t next = lo + (int64_t)(m - 1) * step + 1;
    const int64_t end = lo + (int64_t)m * step;
    len = (end < lo + len ? end : lo + len) - next;
    lo = next;
  }
  return lo;
}

// out row `r` (scaled, rounded once), added to what is there if asked for.
template <int V>
__device__ __forceinline__ void write_row(const EmbeddingGradArgs& a, const Columns<V>& at, int64_t r,
                                          const float (&acc)[V]) {
  float v[V];
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = acc[e] * a.scale;
  int64_t o = r * a.out_stride + at.c;
  if (a.accumulate && at.shift > 0) {
    // an element shared with another thread is added once, by its owner
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float old[1];
      if (e < at.shift) continue;
      load_part<1>(a.out, a.out_type, o + e, 1, old);
      old[0] = __builtin_fmaf(acc[e], a.scale, old[0]);
      store_part<1>(a.out, a.out_type, o + e, 1, old);
    }
    return;
  }
  if (a.accumulate) {
    load_part<V>(a.out, a.out_type, o, at.tiny ? at.D : V, v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = __builtin_fmaf(acc[e], a.scale, v[e]);
  }
  store_part<V>(a.out, a.out_type, o, at.tiny ? at.D : V, v);
}

// Clears the table, 16 bytes a thread: neighbouring blocks write neighbouring
// bytes, which the memory takes fastest (100,000 x 4096 f32 alone 217 us, 7.5 TB/s;
// blocks of eight rows each that leave out the rows a token asked for, found
// among the sorted IDs, 253 us, though they write 6 percent less).  A table
// larger than the caches is stored past them: the gradient rows read next need
// not wait then for what is cleared to leave the caches (16,384 x 4096 bf16 into
// this table 329 us and 299, 12,000 x 2048 into 50,000 rows 108 and 99; 8192 x
// 2048 into 20,000 rows, 164 MB, 56 and 59).
constexpr int64_t kClearPast = int64_t(1) << 28;   // bytes
// LDS that the clear asks for and does not use, so that a compute unit holds
// four of its blocks: stores past the caches from fewer waves come nearer one
// another (100,000 x 4096 f32 233 us, 252 with eight blocks, 364 with two; 2048
// or 512 blocks that go on to further vectors 377 and 331).
constexpr unsigned kClearLds = 40960;
__host__ __device__ static inline int64_t table_bytes(const EmbeddingGradArgs& a) {
  return a.R * a.D * (a.out_type == GBA_F32 ? 4 : 2);
}
template <bool PAST>
__device__ __forceinline__ void clear_table(const EmbeddingGradArgs& a, int64_t block, int64_t blocks) {
  typedef VecOf<uint16_t, 8>::type vec;
  const int size = a.out_type == GBA_F32 ? 2 : 1;   // in units of 2 bytes
  const bool flat = a.out_stride == a.D;
  const int64_t rows = flat ? 1 : a.R, units = (flat ? a.R : 1) * a.D * size;
  const int64_t per_row = ceil_div(units, 8), total = rows * per_row;
  uint16_t* out = static_cast<uint16_t*>(a.out);
  for (int64_t i = block * blockDim.x + threadIdx.x; i < total; i += blocks * blockDim.x) {
    const int64_t row = flat ? 0 : i / per_row;
    const int64_t c = (i - row * per_row) * 8;
    uint16_t* p = out + row * a.out_stride * size + c;
    if (c + 8 <= units) {
      if constexpr (PAST) __builtin_nontemporal_store(vec{}, reinterpret_cast<vec*>(p));
      else *reinterpret_cast<vec*>(p) = vec{};
    } else {
      for (int e = 0; e < (int)(units - c); ++e) p[e] = 0;
    }
  }
}
template <bool PAST>
__global__ void __launch_bounds__(kEmbBlock)
clear_table_kernel(EmbeddingGradArgs a) {
  clear_table<PAST>(a, blockIdx.x, gridDim.x);
}

// The sort of a few tokens, in one launch: a token's place is the number of
// tokens with a smaller ID, and of those before it with the same.  A block
// places 64 tokens, a lane each; its waves share out the tokens they are
// compared with, which come through the scalar cache.  Bound by the
// comparisons, n^2 of them: with 16 waves 2000 tokens 8 us, 4000 12, 8000 16,
// where the radix sort's two or three launches take 20 to 27.  Whole calls in
// us, the radix sort and this: 2000 tokens 26 and 21, 4500 of 17-bit IDs 28.7
// and 26.9, of 27-bit IDs 34.8 and 26.7, 6000 29.2 and 29.4, 35.4 and 29.2, 8192
// 29.7 and 31.4, of 21-bit IDs 31.9 and 31.4, of 27-bit IDs 36.5 and 31.9.
//
// The blocks past those clear the table, which does not wait for the sort
// then: with a table to clear the comparisons take the time of a launch that
// is bound by memory, and more tokens than that are sorted this way.
// Fewer waves a block take longer to compare (16,384 tokens 55 us with 8 and
// 100 with 4) but leave the clear more of the chip, so the block's size goes
// by the bytes to clear per token.  Whole calls in us, the radix sort and 16, 8
// and 4 waves: 16,384 tokens and 1638 MB 299 302 277 268, 410 MB 100 97 89 115,
// 205 MB 68 69 71 113; 8192 and 819 MB 158 144 136 135, 205 MB 59 50 48 63, 82 MB
// 41 34 43 61; 6000 and 205 MB 56 46 44 45, 82 MB 38 30 32 46.
// The comparisons go by the square of the tokens and pass the clear within a
// doubling of 16,384: the radix sort and this, 1638 MB, 16,384 tokens 282 and 268,
// 20,000 293 and 280, 24,576 306 and 299, 32,768 325 and 329, 49,152 363 and 475;
// 410 MB 111 and 105, 20,000 118.6 and 117.9, 24,576 129 and 148.  (A table of
// several GB is cleared faster by a launch of its own: 6554 MB, 16,384 tokens 1005
// and 1079.)
constexpr int64_t kRankMost = 6144, kRankMostWide = 8192, kRankMostClearing = 16384;
constexpr int64_t kRankWideRows = int64_t(1) << 18;   // IDs of more than two 9-bit digits
// (A table to clear makes it pay to 8192 for any IDs: into 30,000 x 32, 6000
// tokens 23.6 and 22.6, into 200,000 x 32, 8192 29.0 and 26.5.)
// Threads of a block, 0: the radix sort.  (Few tokens and a table that the
// caches hold: 509 tokens and 16 MB 14.8 us with 16 waves, 16.0 with 8; 1500 and
// 80 MB 24.9 and 26.1 with 4.)
static int rank_block(const EmbeddingGradArgs& a, bool clear) {
  const int64_t bytes = clear ? table_bytes(a) : 0, per_token = bytes / a.n;
  if (a.n > kRankMostClearing) return 0;
  if (a.n > 4096 || bytes >= kClearPast) {
    if (per_token >= 40000) return 256;
    if (per_token >= 20000) return 512;
  }
  return a.n <= (clear || a.R > kRankWideRows ? kRankMostWide : kRankMost) || per_token >= 12000 ? 1024 : 0;
}
template <int BLOCK, bool PAST>
__global__ void __launch_bounds__(BLOCK)
rank_kernel(const int64_t* __restrict__ ids, int n, int64_t R, uint32_t* __restrict__ keys, uint32_t* __restrict__ vals,
            int32_t* err, int rank_blocks, EmbeddingGradArgs a) {
  constexpr int WAVES = BLOCK / kWave;
  __shared__ uint32_t s_count[WAVES][kWave];
  if ((int)blockIdx.x >= rank_blocks) {
    clear_table<PAST>(a, (int64_t)blockIdx.x - rank_blocks, (int64_t)gridDim.x - rank_blocks);
    return;
  }
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int i0 = (int)blockIdx.x * kWave, i = i0 + lane;
  // by the low words: an ID outside the table is reported, and where it is
  // sorted does not matter
  const int64_t id = ids[i < n ? i : n - 1];
  const uint32_t mine = (uint32_t)id;
  const int share = (n + WAVES - 1) / WAVES;
  const int j0 = w * share < n ? w * share : n, j1 = j0 + share < n ? j0 + share : n;
  const int before = i0 < j1 ? (i0 > j0 ? i0 : j0) : j1;
  const int after = i0 + kWave < j1 ? (i0 + kWave > j0 ? i0 + kWave : j0) : j1;
  uint32_t count = 0;
  constexpr int U = 16;
  int j = j0;
  for (; j + U <= before; j += U) {   // before the block's tokens: the same ID comes first
    uint32_t k[U];
#pragma unroll
    for (int u = 0; u < U; ++u) k[u] = (uint32_t)ids[j + u];
#pragma unroll
    for (int u = 0; u < U; ++u) count += k[u] <= mine ? 1u : 0u;
  }
  for (; j < before; ++j) count += (uint32_t)ids[j] <= mine ? 1u : 0u;
  for (; j < after; ++j) {
    const uint32_t k = (uint32_t)ids[j];
    count += k < mine || (k == mine && j < i) ? 1u : 0u;
  }
  for (; j + U <= j1; j += U) {
    uint32_t k[U];
#pragma unroll
    for (int u = 0; u < U; ++u) k[u] = (uint32_t)ids[j + u];
#pragma unroll
    for (int u = 0; u < U; ++u) count += k[u] < mine ? 1u : 0u;
  }
  for (; j < j1; ++j) count += (uint32_t)ids[j] < mine ? 1u : 0u;
  s_count[w][lane] = count;
  __syncthreads();
  if (w != 0 || i >= n) return;
  uint32_t place = 0;
#pragma unroll
  for (int k = 0; k < WAVES; ++k) place += s_count[k][lane];
  const bool in = (uint64_t)id < (uint64_t)R;
  if (!in) raise_error(err, GBA_DERR_ID_RANGE);
  keys[place] = in ? mine : 0u;
  vals[place] = (uint32_t)i;
}

// ROWS: one row per distinct ID (else the whole table).
//
// A lane group leaves at most two sums that are not finished: `head`, of an ID
// that began before its first position, and `tail`, of one that begins in the
// group and goes on after it.  What an ID gets from the groups after the one
// it begins in is the sum of their heads, up to the first that does not go on
// (`open`) into its next group: a suffix scan over the wave's groups in
// registers, then over the block's waves through LDS.
//
// Bound by the gradient rows' bytes where rows are wide (16,384 x 4096 bf16 into
// a cleared f32 table 37 us, 131 MB read and 60 written at 5.2 TB/s), by the
// latency of a group's batches of random rows where they are narrow (256,000 x
// 32 14 us, 28 MB).  Positions, not IDs, are what is shared out, so this launch
// takes no longer for a token that is half of the batch (the join does, below).
// Added to a table instead of cleared into one: 16,384 x 4096 bf16 with 4956
// distinct IDs 71 us, 49 of them here (a floor of 43, the rows read and written),
// 256,000 x 32 with 58,000 46, 15 of them here.
//
// ONE: one block per column slice for at most kOneMost tokens, which it sorts
// itself.
template <typename T, int LPR, bool ROWS, bool ONE>
__global__ void __launch_bounds__(kEmbBlock)
embedding_grad_kernel(EmbeddingGradArgs a, GradScratch g) {
  constexpr int V = kVec<T>;
  constexpr int G = kEmbBlock / LPR;
  constexpr int kGroups = kWave / LPR;           // lane groups of a wave
  constexpr int POS = G * 32 < kMaxPos ? G * 32 : kMaxPos;   // most positions of the block
  typedef typename VecOf<T, V>::type vec;
  __shared__ uint32_t sk[POS];                   // the block's keys
  __shared__ uint32_t sv[POS];                   // ... their tokens
  __shared__ uint32_t srun[ROWS ? POS : 1];      // ... their rows of the output
  __shared__ float s_head[kEmbWaves][LPR * V];   // what the waves' first groups give to an ID of an earlier wave
  __shared__ uint32_t s_open[kEmbWaves];         // ... and whether it goes on into the next wave
  __shared__ uint32_t s_scan[kEmbWaves + 1];
  __shared__ uint32_t s_group[kEmbWaves];
  __shared__ uint32_t s_pad;

  const unsigned block = blockIdx.x / g.slices;
  const int slice = (int)(blockIdx.x - block * g.slices);
  const int S = g.span;
  const int64_t b0 = (int64_t)block * g.pos;
  const int cnt = (int)(a.n - b0 < g.pos ? a.n - b0 : g.pos);
  const bool padded = a.padding >= 0 && a.padding < a.R;
  const uint32_t pad = (uint32_t)a.padding;
  // keys before the block and after it (there is none: no key is equal)
  const bool has_prev = !ONE && b0 > 0, has_next = !ONE && b0 + cnt < a.n;
  const uint32_t prev = has_prev ? a.keys[b0 - 1] : 0u;
  const uint32_t next = has_next ? a.keys[b0 + cnt] : 0u;
  if constexpr (ONE) {
    // by the number of smaller IDs and of the same before it
    const int i = threadIdx.x;
    const int64_t id = i < cnt ? a.ids[i] : 0;
    const bool in = (uint64_t)id < (uint64_t)a.R;
    const uint32_t key = in ? (uint32_t)id : 0u;
    if (!in) raise_error(a.err, GBA_DERR_ID_RANGE);
    if (i < cnt) sv[i] = key;
    if (i == 0) s_pad = 0u;
    __syncthreads();
    int place = 0;
#pragma unroll 8
    for (int j = 0; j < cnt; ++j) place += sv[j] < key || (sv[j] == key && j < i) ? 1 : 0;
    __syncthreads();
    if (i < cnt) {
      const bool hide = padded && key == pad;
      if (hide) s_pad = 1u;
      sk[place] = key;
      sv[place] = hide ? 0u : (uint32_t)i;
    }
  } else {
    for (int i = threadIdx.x; i < cnt; i += kEmbBlock) {
      const uint32_t key = a.keys[b0 + i], val = a.vals[b0 + i];
      sk[i] = key;
      sv[i] = padded && key == pad ? 0u : val;   // (a padding token's row is not needed: one that is near)
    }
  }
  const bool tiled = !ONE && g.heads.tile_prefix != nullptr;
  if (ROWS) {
    // run heads in the block's tile before the block, or in all of a few tokens
    constexpr int kEarlier = (int)(kRunTile / kEmbBlock);
    const int64_t tile = b0 / kRunTile;
    uint32_t earlier = 0;
    for (int64_t t = tiled ? tile : 0; t <= tile; ++t) {
#pragma unroll
      for (int k = 0; k < kEarlier; ++k) {
        const int64_t q = t * kRunTile + k * kEmbBlock + threadIdx.x;
        if (q < b0) earlier += (q == 0 || a.keys[q] != a.keys[q - 1]) ? 1u : 0u;
      }
    }
    if (tiled) run_base(g.heads, tile, s_group);
    earlier = wave_sum(earlier);
    if (lane_id() == 0) s_scan[threadIdx.x / kWave] = earlier;
    // does the padding ID occur?  Its run is not numbered.
    if (!ONE && padded && threadIdx.x < kWave) {
      const int64_t at = wave_lower_bound(a.keys, a.n, pad);
      if (threadIdx.x == 0) s_pad = at < a.n && a.keys[at] == pad ? 1u : 0u;
    }
  }
  __syncthreads();

  const int w = threadIdx.x / kWave;
  const int grp = threadIdx.x / LPR, gl = threadIdx.x % LPR;
  const Columns<V> at(slice * (LPR * V) + gl * V, a.D);
  const int first = grp * S, end = first + S < cnt ? first + S : cnt;
  const T* grad = static_cast<const T*>(a.grad) + at.c;
  auto load_batch = [&](int p, vec (&v)[kRows]) {
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      uint32_t row = sv[p + u < end ? p + u : end - 1];   // past the end the last row again
      if constexpr (LPR == kWave) row = __builtin_amdgcn_readfirstlane(row);
      const T* src = grad + (int64_t)row * a.grad_stride;
      if (at.tiny) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[u][e] = e < at.D ? src[e] : (T)0.0f;
      } else {
        v[u] = *reinterpret_cast<const vec*>(src);
      }
    }
  };
  vec v[kRows], ahead[kRows];
  const bool busy = at.on && first < end;
  if (busy) load_batch(first, v);   // in flight while the rows are numbered

  if (ROWS) {
    uint32_t base = tiled ? g.heads.tile_prefix[b0 / kRunTile] + run_base_sum(s_group) : 0u;
#pragma unroll
    for (int k = 0; k < kEmbWaves; ++k) base += s_scan[k];
    __syncthreads();
    constexpr int PER = POS >= kEmbBlock ? POS / kEmbBlock : 1;
    const int p0 = threadIdx.x * PER;
    uint32_t h[PER], sum = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int p = p0 + k;
      h[k] = p < cnt && (p == 0 ? !has_prev || sk[0] != prev : sk[p] != sk[p - 1]) ? 1u : 0u;
      sum += h[k];
    }
    uint32_t all;
    uint32_t run = base + block_exclusive_scan<kEmbBlock>(sum, s_scan, &all);
    const uint32_t hidden = padded ? s_pad : 0u;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int p = p0 + k;
      if (p >= cnt) break;
      run += h[k];
      const uint32_t key = sk[p];
      const uint32_t r = run - 1 - (hidden && key > pad ? 1u : 0u);
      srun[p] = r;
      if (slice == 0) {
        if (h[k] && !(padded && key == pad)) a.unique_ids[r] = (int64_t)key;
        if (b0 + p == a.n - 1) *a.num_unique = (int64_t)run - hidden;
      }
    }
    __syncthreads();
  }

  auto next_is = [&](int p, uint32_t key) { return p + 1 < cnt ? sk[p + 1] == key : has_next && next == key; };
  auto prev_is = [&](int p, uint32_t key) { return p > 0 ? sk[p - 1] == key : has_prev && prev == key; };
  auto out_row = [&](int p) { return ROWS ? (int64_t)srun[p] : (int64_t)sk[p]; };

  // Bit i of a group's word: the ID at its position i ends there.  The
  // positions of a wave's groups are adjacent: 64 a ballot.
  uint32_t ends = 0;
  {
    const int w0 = w * kGroups * S;
    const int mine = (grp % kGroups) * S;
    for (int k = 0; k < kGroups * S; k += kWave) {
      const int p = w0 + k + lane_id();
      const bool stop = k + lane_id() < kGroups * S && p < cnt && !next_is(p, sk[p]);
      const uint64_t m = __ballot(stop);
      if (mine >= k && mine < k + kWave) ends = (uint32_t)(m >> (mine - k));
    }
  }

  float head[V] = {}, tail[V] = {};
  const bool some = first < end;
  const bool has_head = some && prev_is(first, sk[some ? first : 0]);
  if (busy) {
    float acc[V] = {};
    bool begins = !has_head;
    for (int p = first; p < end; p += kRows) {
      if (p + kRows < end) load_batch(p + kRows, ahead);
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int q = p + u;
        if (q >= end) break;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += (float)v[u][e];
        if (!(ends >> (q - first) & 1u)) continue;
        const uint32_t key = sk[q];
        if (!begins) {
#pragma unroll
          for (int e = 0; e < V; ++e) head[e] = acc[e];
        } else if (!(padded && key == pad)) {
          write_row<V>(a, at, out_row(q), acc);
        }
        begins = true;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.0f;
      }
      if (p + kRows < end) {
#pragma unroll
        for (int u = 0; u < kRows; ++u) v[u] = ahead[u];
      }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if (begins) tail[e] = acc[e];
      else head[e] = acc[e];
    }
  }
  const uint32_t key = sk[some ? end - 1 : 0];
  const bool goes_on = some && !(ends >> (end - 1 - first) & 1u);
  const uint32_t full = some ? ends & (uint32_t)((1ull << (end - first)) - 1) : 0u;
  bool open = has_head && goes_on && full == 0;   // the group's only ID, from before it to after it
  const bool has_tail = goes_on && !open;

  // head becomes the sum of the heads from this group on
#pragma unroll
  for (int off = 1; off < kGroups; off <<= 1) {
    const bool here = grp % kGroups + off < kGroups;
    const bool then = __shfl_down((int)open, off * LPR, kWave) != 0;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float more = __shfl_down(head[e], off * LPR, kWave);
      head[e] += open && here ? more : 0.0f;
    }
    if (here) open = open && then;
  }
  if (grp % kGroups == 0) {
#pragma unroll
    for (int e = 0; e < V; ++e) s_head[w][gl * V + e] = head[e];
    if (gl == 0) s_open[w] = open ? 1u : 0u;
  }
  // the group after this one, where it is in the wave (every lane takes part
  // in the exchange: a lane that does not would give 0)
  float after[V];
  const bool last_group = grp % kGroups == kGroups - 1;
  const int next_open = kGroups > 1 ? __shfl_down((int)open, LPR, kWave) : 0;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float more = kGroups > 1 ? __shfl_down(head[e], LPR, kWave) : 0.0f;
    after[e] = last_group ? 0.0f : more;
  }
  const bool after_open = last_group || next_open != 0;
  __syncthreads();
  if (!at.on || !some) return;

  // adds the heads of the waves after this one; true: they go on past the block
  auto add_waves = [&](float (&acc)[V]) {
    for (int k = w + 1; k < kEmbWaves; ++k) {
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] += s_head[k][gl * V + e];
      if (!s_open[k]) return false;
    }
    return true;
  };
  float* piece = g.pieces + (int64_t)block * 2 * a.D + at.c;
  if (grp == 0 && has_head && !(padded && sk[0] == pad)) {
    // the block's first ID began in an earlier block
    if (open) add_waves(head);
    store_part<float, V>(piece, at.tiny ? at.D : V, head);
  }
  if (!has_tail || (padded && key == pad)) return;
  bool past = has_next && next == key && end == cnt;   // past the block
  if (end < cnt) {
#pragma unroll
    for (int e = 0; e < V; ++e) tail[e] += after[e];
    past = after_open && add_waves(tail);
  }
  if (past) {
    store_part<float, V>(piece + a.D, at.tiny ? at.D : V, tail);
    if (ROWS && slice == 0 && gl == 0) g.tail_run[block] = srun[end - 1];
  } else {
    write_row<V>(a, at, out_row(end - 1), tail);
  }
}

// The IDs that cross blocks: by the block in which each begins.  A launch that
// does little (3 to 5 us): most blocks compare two keys and end.  Bound by the
// one block of a very frequent ID's column slice, whose lane groups read its
// pieces in turn: 234,375 x 512 bf16 5 us, 44 with an ID that is a fifth of the
// tokens, 86 with one that is half (whole calls 195, 217, 237, as there are fewer
// rows to write then; 256,000 x 32 51, 53, 53).
template <int V, int LPR, bool ROWS>
__global__ void __launch_bounds__(kEmbBlock)
embedding_grad_join_kernel(EmbeddingGradArgs a, GradScratch g) {
  constexpr int G = kEmbBlock / LPR;
  __shared__ float s_sum[G][LPR * V];
  const int64_t b = blockIdx.x / g.slices;
  const int slice = (int)(blockIdx.x - b * g.slices);
  const int pos = g.pos;
  const int64_t first = (b + 1) * pos;           // the next block's first position (< n)
  const uint32_t key = a.keys[first - 1];
  if (a.keys[first] != key) return;
  if (b > 0 && a.keys[b * pos] == key && a.keys[b * pos - 1] == key) return;   // began earlier
  if (a.padding >= 0 && (int64_t)key == a.padding) return;
  // blocks after b whose first key it is
  int64_t m = 1;
  for (;;) {
    const int64_t j = b + 1 + m + lane_id();
    const uint64_t same = __ballot(j < (int64_t)g.blocks && a.keys[j * pos] == key);
    const int run = same == ~0ull ? kWave : __ffsll((unsigned long long)~same) - 1;
    m += run;
    if (run < kWave) break;
  }
  const int grp = threadIdx.x / LPR, gl = threadIdx.x % LPR;
  const Columns<V> at(slice * (LPR * V) + gl * V, a.D);
  const int count = at.tiny ? at.D : V;
  float acc[V] = {};
  if (at.on) {
#pragma unroll 4
    for (int64_t j = grp; j < m; j += G) {
      float v[V];
      load_part<float, V>(g.pieces + (b + 1 + j) * 2 * a.D + at.c, count, v);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] += v[e];
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) s_sum[grp][gl * V + e] = acc[e];
  __syncthreads();
  if (grp != 0 || !at.on) return;
  load_part<float, V>(g.pieces + (b * 2 + 1) * a.D + at.c, count, acc);
  const int used = m < G ? (int)m : G;
  for (int j = 0; j < used; ++j) {
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] += s_sum[j][gl * V + e];
  }
  const int64_t row = ROWS ? (int64_t)g.tail_run[b] : (int64_t)key;
  if (row < (ROWS ? a.n : a.R)) write_row<V>(a, at, row, acc);   // always, when the numbering is consistent
}

constexpr int64_t kCountMost = 4096;   // tokens whose run heads every block counts
__global__ void no_rows_kernel(int64_t* __restrict__ num_unique) { *num_unique = 0; }

// Positions of a lane group: the most a block's kMaxPos leave, 32 at most, or
// fewer (kRows at least) while that makes less than kWavesWanted waves.  (With
// batches of 8 rows and twice to four times the waves: 2000 rows of 256 bf16
// 21 us and 20, 400,000 of 64 80 and 78, 509 of 1001 16.5 and 15.1.)
constexpr int64_t kWavesWanted = 1024;
static int most_span(int lpr) { return lpr < 8 ? 4 * lpr : 32; }
static int group_span(int64_t n, int lpr, int64_t slices) {
  int s = most_span(lpr);
  while (s > kRows && n * slices * lpr < kWavesWanted * kWave * s) s >>= 1;
  return s;
}

// A few tokens in one launch, as far as the spans stay at kOneSpan: 4 tokens
// of 64 floats 8.3 us and 10.9 with a launch that sorts, 32 of 2048 9.1 and 13.5
// (60 in spans of 16 13.0 and 13.1; 200 of 64 14.3 and 13.4: the comparisons of
// one block take longer than those of many).
constexpr int kOneMost = kWave, kOneSpan = 8;
static bool one_block(int64_t n, int lpr) {
  return n <= kOneMost && n <= (int64_t)kOneSpan * kEmbBlock / lpr;
}

struct GradLayout {
  size_t off_pieces, off_tail, off_tile, off_group, bytes;
};
// Room for every size up to n and any element type: the most blocks that a
// size up to n has at each span.
static GradLayout grad_layout(int64_t n, int32_t D) {
  int64_t blocks = 1;
  for (int v = kVec<float>; v <= kVec<bf16_t>; v += v) {
    const int lpr = lanes_for(D, v);
    const int64_t slices = ceil_div(D, (int64_t)lpr * v);
    for (int s = most_span(lpr);; s >>= 1) {
      int64_t most = n;
      if (s < most_span(lpr)) most = std::min(n, ceil_div(kWavesWanted * kWave * 2 * s, slices * lpr));
      blocks = std::max(blocks, ceil_div(most, kEmbBlock / lpr * s));
      if (s <= kRows) break;
    }
  }
  const int64_t tiles = ceil_div(std::max<int64_t>(n, 1), kRunTile);
  GradLayout L{};
  size_t o = 0;
  L.off_pieces = o; o += align_up((size_t)blocks * 2 * (size_t)D * sizeof(float));
  L.off_tail = o;   o += align_up((size_t)blocks * 4);
  L.off_tile = o;   o += align_up((size_t)tiles * 4);
  // (the groups grow fourfold at 4096 tiles: their counts keep the room of the smaller sizes)
  L.off_group = o;  o += align_up((size_t)std::max(run_groups(n), std::min<int64_t>(tiles, 1024)) * 4);
  L.bytes = o;
  return L;
}

// The sorted IDs' part of the workspace.
static size_t sort_bytes(int64_t n, int64_t R) {
  return std::max(align_up(plan_sort(n, R).bytes), 2 * align_up((size_t)std::min(n, kRankMostClearing) * 4));
}

size_t embedding_grad_workspace_bytes(int64_t n, int32_t D, int64_t R) {
  return sort_bytes(n, R) + grad_layout(n, D).bytes;
}

template <typename T, int LPR, bool ROWS>
static hipError_t grad_as(const EmbeddingGradArgs& a, GradScratch g, hipStream_t stream) {
  constexpr int V = kVec<T>;
  g.slices = (int)ceil_div(a.D, LPR * V);
  g.span = group_span(a.n, LPR, g.slices);
  if (a.ids) {
    g.span = kRows;
    while (kEmbBlock / LPR * g.span < a.n) g.span <<= 1;
    g.pos = kEmbBlock / LPR * g.span;
    g.blocks = 1;
    hipLaunchKernelGGL((embedding_grad_kernel<T, LPR, ROWS, true>), dim3((unsigned)g.slices), dim3(kEmbBlock), 0,
                       stream, a, g);
    return hipGetLastError();
  }
  g.pos = kEmbBlock / LPR * g.span;
  const int64_t blocks = ceil_div(a.n, g.pos);
  g.blocks = (unsigned)blocks;
  const int64_t grid = blocks * g.slices;
  if (grid > kMostBlocks) return hipErrorInvalidValue;
  hipLaunchKernelGGL((embedding_grad_kernel<T, LPR, ROWS, false>), dim3((unsigned)grid),
                     dim3(kEmbBlock), 0, stream, a, g);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || blocks == 1) return e;
  hipLaunchKernelGGL((embedding_grad_join_kernel<V, LPR, ROWS>), dim3((unsigned)((blocks - 1) * g.slices)),
                     dim3(kEmbBlock), 0, stream, a, g);
  return hipGetLastError();
}

template <typename T, bool ROWS>
static hipError_t grad_of(const EmbeddingGradArgs& a, const GradScratch& g, hipStream_t stream) {
  switch (lanes_for(a.D, kVec<T>)) {
    case 1: return grad_as<T, 1, ROWS>(a, g, stream);
    case 2: return grad_as<T, 2, ROWS>(a, g, stream);
    case 4: return grad_as<T, 4, ROWS>(a, g, stream);
    case 8: return grad_as<T, 8, ROWS>(a, g, stream);
    case 16: return grad_as<T, 16, ROWS>(a, g, stream);
    case 32: return grad_as<T, 32, ROWS>(a, g, stream);
    default: return grad_as<T, 64, ROWS>(a, g, stream);
  }
}

hipError_t launch_embedding_grad(const int64_t* ids, EmbeddingGradArgs a, void* ws, int32_t* err, hipStream_t stream) {
  const bool rows = a.num_unique != nullptr;
  const bool clear = !rows && !a.accumulate;
  if (rows && a.n == 0) {
    hipLaunchKernelGGL(no_rows_kernel, dim3(1), dim3(1), 0, stream, a.num_unique);
    return hipGetLastError();
  }
  // A table to clear takes a launch before the one that adds up; sorting there
  // costs none, so one block pays where it saves the join: 20 rows of 2048 into
  // 1000 12.4 us and 10.3, 32 into 10,000 21.9 and 20.1.
  const int V = a.grad_type == GBA_F32 ? kVec<float> : kVec<bf16_t>, lpr = lanes_for(a.D, V);
  const bool joins = a.n > (int64_t)kEmbBlock / lpr * group_span(a.n, lpr, ceil_div(a.D, lpr * V));
  const bool one = a.n > 0 && one_block(a.n, lpr) && (!clear || (joins && table_bytes(a) < kClearPast));
  a.ids = one ? ids : nullptr;
  a.err = err;
  const int64_t vecs = clear ? a.R * ceil_div((int64_t)a.D * (a.out_type == GBA_F32 ? 4 : 2), 16) : 0;
  char* base = static_cast<char*>(ws);
  hipError_t e;
  const int size = a.n > 0 && !one ? rank_block(a, clear) : 0;
  if (size > 0) {
    uint32_t* keys = reinterpret_cast<uint32_t*>(base);
    uint32_t* vals = reinterpret_cast<uint32_t*>(base + align_up((size_t)a.n * 4));
    const int64_t ranks = ceil_div(a.n, kWave), clears = std::min(ceil_div(vecs, size), kMaxGrid);
    const dim3 grid((unsigned)(ranks + clears)), block((unsigned)size);
    const bool past = clear && table_bytes(a) >= kClearPast;
    const auto kernel = size == 256   ? (past ? rank_kernel<256, true> : rank_kernel<256, false>)
                        : size == 512 ? (past ? rank_kernel<512, true> : rank_kernel<512, false>)
                                      : (past ? rank_kernel<1024, true> : rank_kernel<1024, false>);
    hipLaunchKernelGGL(kernel, grid, block, 0, stream, ids, (int)a.n, a.R, keys, vals, err, (int)ranks, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    a.keys = keys;
    a.vals = vals;
  } else {
    if (clear) {
      const dim3 grid((unsigned)std::min(ceil_div(vecs, kEmbBlock), kMaxGrid)), block(kEmbBlock);
      if (table_bytes(a) >= kClearPast) hipLaunchKernelGGL(clear_table_kernel<true>, grid, block, kClearLds, stream, a);
      else hipLaunchKernelGGL(clear_table_kernel<false>, grid, block, 0, stream, a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.n == 0) return hipSuccess;
    if (!one) {
      e = launch_sort_ids(ids, a.n, a.R, plan_sort(a.n, a.R), ws, &a.keys, &a.vals, err, stream);
      if (e != hipSuccess) return e;
    }
  }
  const GradLayout L = grad_layout(a.n, a.D);
  base += sort_bytes(a.n, a.R);
  GradScratch g{};
  g.pieces = reinterpret_cast<float*>(base + L.off_pieces);
  g.tail_run = reinterpret_cast<uint32_t*>(base + L.off_tail);
  if (rows) {
    // (of a few tokens the blocks count the run heads before them themselves:
    // 4500 tokens 28.2 us, 28.7 with a launch that counts for them, 6000 30.1 and
    // 29.2)
    if (a.n > kCountMost) {
      e = launch_run_heads(a.keys, a.n, reinterpret_cast<uint32_t*>(base + L.off_tile),
                           reinterpret_cast<uint32_t*>(base + L.off_group), &g.heads, stream);
      if (e != hipSuccess) return e;
    }
    if (a.grad_type == GBA_F32) return grad_of<float, true>(a, g, stream);
    if (a.grad_type == GBA_BF16) return grad_of<bf16_t, true>(a, g, stream);
    return grad_of<f16_t, true>(a, g, stream);
  }
  if (a.grad_type == GBA_F32) return grad_of<float, false>(a, g, stream);
  if (a.grad_type == GBA_BF16) return grad_of<bf16_t, false>(a, g, stream);
  return grad_of<f16_t, false>(a, g, stream);
}

}  // namespace gba
