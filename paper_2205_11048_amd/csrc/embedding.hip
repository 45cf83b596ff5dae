// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// The gradient: the tokens are sorted by ID (the push path's stable sort), and
// the sorted list is cut into blocks of positions whatever the IDs, so that a
// frequent ID's tokens are shared among many lane groups.  A lane group adds
// up the gradient rows of its positions; an ID that begins and ends inside the
// group goes straight to the output, what crosses a group's edge is joined in
// LDS by the group where the ID begins, and what crosses a block's edge by a
// second launch, through 32-bit partial rows.  Every sum has one order, so the
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

__host__ __device__ static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

// Lanes that share a row slice of V elements each: a power of two, up to a wave.
static int lanes_for(int32_t D, int V) {
  int l = 1;
  while (l < kWave && l * V < D) l <<= 1;
  return l;
}

// ---------------------------------------------------------------- lookup
// A vector of V elements per thread and step.
template <typename T, typename O, int V>
__global__ void __launch_bounds__(kEmbBlock)
lookup_kernel(LookupArgs a) {
  const int64_t per_row = ceil_div(a.D, V);
  const int64_t total = a.n * per_row;
  for (int64_t i = (int64_t)blockIdx.x * kEmbBlock + threadIdx.x; i < total; i += (int64_t)gridDim.x * kEmbBlock) {
    const int64_t row = i / per_row;
    const int c = (int)(i - row * per_row) * V;
    const int64_t id = a.ids[row];
    const bool ok = (uint64_t)id < (uint64_t)a.R;
    float v[V] = {};
    if (ok) load_part<T, V>(static_cast<const T*>(a.table) + id * a.table_stride + c, a.D - c, v);
    else if (c == 0) raise_error(a.err, GBA_DERR_ID_RANGE);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] *= a.scale;
    store_part<O, V>(static_cast<O*>(a.out) + row * a.out_stride + c, a.D - c, v);
  }
}

template <typename T, typename O>
static hipError_t lookup_as(const LookupArgs& a, hipStream_t stream) {
  constexpr int V = kVec<T> > kVec<O> ? kVec<T> : kVec<O>;
  const int64_t blocks = std::min(ceil_div(a.n * ceil_div(a.D, V), kEmbBlock), kMaxGrid);
  hipLaunchKernelGGL((lookup_kernel<T, O, V>), dim3((unsigned)blocks), dim3(kEmbBlock), 0, stream, a);
  return hipGetLastError();
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
// Positions of a lane group and of a block, for lpr lanes per row slice.
constexpr int group_span(int lpr) { return lpr <= 8 ? 4 * lpr : 32; }
constexpr int block_span(int lpr) { return kEmbBlock / lpr * group_span(lpr); }
static_assert(block_span(1) == 1024 && block_span(8) == 1024 && block_span(64) == 128, "spans divide a run tile");

struct GradScratch {
  RunHeads heads;          // one row per distinct ID: where the blocks' numbering begins
  float* pieces;           // [blocks][2][D]: what the block's first ID adds to an ID of an earlier block, and the
                           // block's part of an ID that begins in it and goes on in the next
  uint32_t* tail_run;      // [blocks] the row of that second ID (one row per distinct ID)
};

// The first position whose key is not below `key` in keys[0, n): 64 probes a
// step, by one wave.
__device__ __forceinline__ int64_t wave_lower_bound(const uint32_t* __restrict__ keys, int64_t n, uint32_t key) {
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
__device__ __forceinline__ void write_row(const EmbeddingGradArgs& a, int64_t r, int c, const float (&acc)[V]) {
  float v[V];
  const int64_t at = r * a.out_stride + c;
  if (a.accumulate) {
    load_part<V>(a.out, a.out_type, at, a.D - c, v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = __builtin_fmaf(acc[e], a.scale, v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = acc[e] * a.scale;
  }
  store_part<V>(a.out, a.out_type, at, a.D - c, v);
}

// ROWS: one row per distinct ID (else the whole table).
template <typename T, int LPR, bool ROWS>
__global__ void __launch_bounds__(kEmbBlock)
embedding_grad_kernel(EmbeddingGradArgs a, GradScratch g) {
  constexpr int V = kVec<T>;
  constexpr int G = kEmbBlock / LPR;
  constexpr int S = group_span(LPR);
  constexpr int POS = block_span(LPR);
  constexpr int kRows = 8;                       // rows in flight per lane group
  static_assert(S % 4 == 0, "whole batches");
  __shared__ uint32_t sk[POS];                   // the block's keys
  __shared__ uint32_t sv[POS];                   // ... their tokens
  __shared__ uint32_t srun[ROWS ? POS : 1];      // ... their rows of the output
  __shared__ float s_piece[2][G][LPR * V];       // what crosses the groups' edges
  __shared__ uint32_t s_scan[kEmbWaves + 1];
  __shared__ uint32_t s_group[kEmbWaves];
  __shared__ uint32_t s_pad;

  const int64_t b0 = (int64_t)blockIdx.x * POS;
  const int cnt = (int)(a.n - b0 < POS ? a.n - b0 : POS);
  const bool padded = a.padding >= 0 && a.padding < a.R;
  const uint32_t pad = (uint32_t)a.padding;
  // keys before the block and after it (there is none: no key is equal)
  const bool has_prev = b0 > 0, has_next = b0 + cnt < a.n;
  const uint32_t prev = has_prev ? a.keys[b0 - 1] : 0u;
  const uint32_t next = has_next ? a.keys[b0 + cnt] : 0u;
  for (int i = threadIdx.x; i < cnt; i += kEmbBlock) {
    sk[i] = a.keys[b0 + i];
    sv[i] = a.vals[b0 + i];
  }
  if (ROWS) {
    // run heads in the block's tile before the block
    constexpr int kEarlier = (int)(kRunTile / kEmbBlock);
    const int64_t tile = b0 / kRunTile;
    uint32_t earlier = 0;
#pragma unroll
    for (int k = 0; k < kEarlier; ++k) {
      const int64_t q = tile * kRunTile + k * kEmbBlock + threadIdx.x;
      if (q < b0) earlier += (q == 0 || a.keys[q] != a.keys[q - 1]) ? 1u : 0u;
    }
    run_base(g.heads, tile, s_group);
    earlier = wave_sum(earlier);
    if (lane_id() == 0) s_scan[threadIdx.x / kWave] = earlier;
    // does the padding ID occur?  Its run is not numbered.
    if (padded && threadIdx.x < kWave) {
      const int64_t at = wave_lower_bound(a.keys, a.n, pad);
      if (threadIdx.x == 0) s_pad = at < a.n && a.keys[at] == pad ? 1u : 0u;
    }
  }
  __syncthreads();
  if (ROWS) {
    uint32_t base = g.heads.tile_prefix[b0 / kRunTile] + run_base_sum(s_group);
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
      if (blockIdx.y == 0) {
        if (h[k] && !(padded && key == pad)) a.unique_ids[r] = (int64_t)key;
        if (b0 + p == a.n - 1) *a.num_unique = (int64_t)run - hidden;
      }
    }
    __syncthreads();
  }

  const int grp = threadIdx.x / LPR, gl = threadIdx.x % LPR;
  const int c = (int)blockIdx.y * (LPR * V) + gl * V;
  const bool on = c < a.D;   // (a group's lanes past the row's end only wait at the barrier)
  const int first = grp * S, end = first + S < cnt ? first + S : cnt;
  auto next_is = [&](int p, uint32_t key) { return p + 1 < cnt ? sk[p + 1] == key : has_next && next == key; };
  auto prev_is = [&](int p, uint32_t key) { return p > 0 ? sk[p - 1] == key : has_prev && prev == key; };
  auto out_row = [&](int p) { return ROWS ? (int64_t)srun[p] : (int64_t)sk[p]; };

  if (on && first < end) {
    const T* grad = static_cast<const T*>(a.grad) + c;
    const int count = a.D - c;
    float acc[V] = {};
    bool begins = !prev_is(first, sk[first]);
    for (int p = first; p < end; p += kRows) {
      float v[kRows][V];
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        // past the end the last row again; a padding token's row is not looked at
        const int q = p + u < end ? p + u : end - 1;
        if (padded && sk[q] == pad) {
#pragma unroll
          for (int e = 0; e < V; ++e) v[u][e] = 0.0f;
        } else {
          load_part<T, V>(grad + (int64_t)sv[q] * a.grad_stride, count, v[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int q = p + u;
        if (q >= end) break;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += v[u][e];
        const uint32_t key = sk[q];
        const bool goes_on = next_is(q, key);
        if (goes_on && q + 1 < end) continue;
        if (!(padded && key == pad)) {
          if (begins && !goes_on) {
            write_row<V>(a, out_row(q), c, acc);
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e) s_piece[begins ? 1 : 0][grp][gl * V + e] = acc[e];
          }
        }
        begins = true;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.0f;
      }
    }
  }
  __syncthreads();
  if (!on || first >= end) return;

  // The sum of s_piece[0] over the groups after `j0` that hold `key`; *last is
  // the last position of the key in the block.
  auto chain = [&](int j0, uint32_t key, float (&acc)[V], int* last) {
    int at = (j0 + 1) * S < cnt ? (j0 + 1) * S : cnt;   // first position not added yet
    for (int j = j0 + 1; at < cnt && sk[at] == key; ++j) {
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] += s_piece[0][j][gl * V + e];
      at = (j + 1) * S < cnt ? (j + 1) * S : cnt;
      if (sk[at - 1] != key) {   // ends inside the group
        *last = -1;
        return;
      }
    }
    *last = at - 1;
  };
  float* piece = g.pieces + (int64_t)blockIdx.x * 2 * a.D + c;
  if (grp == 0 && prev_is(0, sk[0]) && !(padded && sk[0] == pad)) {
    // the block's first ID began in an earlier block
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = s_piece[0][0][gl * V + e];
    int last;
    if (sk[end - 1] == sk[0]) chain(0, sk[0], acc, &last);
    store_part<float, V>(piece, a.D - c, acc);
  }
  const uint32_t key = sk[end - 1];
  if (!next_is(end - 1, key) || (padded && key == pad)) return;
  if (sk[first] == key && prev_is(first, key)) return;   // began in an earlier group
  float acc[V];
#pragma unroll
  for (int e = 0; e < V; ++e) acc[e] = s_piece[1][grp][gl * V + e];
  int last;
  chain(grp, key, acc, &last);
  if (last == cnt - 1 && has_next && next == key) {
    store_part<float, V>(piece + a.D, a.D - c, acc);
    if (ROWS && blockIdx.y == 0 && gl == 0) g.tail_run[blockIdx.x] = srun[end - 1];
  } else {
    write_row<V>(a, out_row(end - 1), c, acc);
  }
}

// The IDs that cross blocks: by the block in which each begins.
template <int V, int LPR, bool ROWS>
__global__ void __launch_bounds__(kEmbBlock)
embedding_grad_join_kernel(EmbeddingGradArgs a, GradScratch g, int pos) {
  constexpr int G = kEmbBlock / LPR;
  __shared__ float s_sum[G][LPR * V];
  const int64_t b = blockIdx.x;
  const int64_t at = (b + 1) * pos;              // the next block's first position (< n)
  const uint32_t key = a.keys[at - 1];
  if (a.keys[at] != key) return;
  if (b > 0 && a.keys[b * pos] == key && a.keys[b * pos - 1] == key) return;   // began earlier
  if (a.padding >= 0 && (int64_t)key == a.padding) return;
  // blocks after b whose first key it is
  int64_t m = 1;
  const int64_t blocks = (a.n + pos - 1) / pos;
  for (;;) {
    const int64_t j = b + 1 + m + lane_id();
    const uint64_t same = __ballot(j < blocks && a.keys[j * pos] == key);
    const int run = same == ~0ull ? kWave : __ffsll((unsigned long long)~same) - 1;
    m += run;
    if (run < kWave) break;
  }
  const int grp = threadIdx.x / LPR, gl = threadIdx.x % LPR;
  const int c = (int)blockIdx.y * (LPR * V) + gl * V;
  const bool on = c < a.D;
  float acc[V] = {};
  if (on) {
    for (int64_t j = grp; j < m; j += G) {
      float v[V];
      load_part<float, V>(g.pieces + (b + 1 + j) * 2 * a.D + c, a.D - c, v);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] += v[e];
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) s_sum[grp][gl * V + e] = acc[e];
  __syncthreads();
  if (grp != 0 || !on) return;
  load_part<float, V>(g.pieces + (b * 2 + 1) * a.D + c, a.D - c, acc);
  const int used = m < G ? (int)m : G;
  for (int j = 0; j < used; ++j) {
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] += s_sum[j][gl * V + e];
  }
  write_row<V>(a, ROWS ? (int64_t)g.tail_run[b] : (int64_t)key, c, acc);
}

__global__ void __launch_bounds__(kEmbBlock)
zero_rows_kernel(EmbeddingGradArgs a) {
  constexpr int V = 4;
  const int64_t per_row = ceil_div(a.D, V);
  const int64_t total = a.R * per_row;
  const float zero[V] = {};
  for (int64_t i = (int64_t)blockIdx.x * kEmbBlock + threadIdx.x; i < total; i += (int64_t)gridDim.x * kEmbBlock) {
    const int64_t row = i / per_row;
    const int c = (int)(i - row * per_row) * V;
    store_part<V>(a.out, a.out_type, row * a.out_stride + c, a.D - c, zero);
  }
}

__global__ void no_rows_kernel(int64_t* __restrict__ num_unique) { *num_unique = 0; }

struct GradLayout {
  size_t off_pieces, off_tail, off_tile, off_group, bytes;
};
// Room for every size up to n and any element type.
static GradLayout grad_layout(int64_t n, int32_t D) {
  // the fewest positions of a block: those of 4-byte elements (the most lanes a row)
  const int64_t blocks = ceil_div(std::max<int64_t>(n, 1), block_span(lanes_for(D, kVec<float>)));
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

size_t embedding_grad_workspace_bytes(int64_t n, int32_t D) { return grad_layout(n, D).bytes; }

template <typename T, int LPR, bool ROWS>
static hipError_t grad_as(const EmbeddingGradArgs& a, const GradScratch& g, hipStream_t stream) {
  constexpr int V = kVec<T>;
  constexpr int POS = block_span(LPR);
  const int64_t blocks = ceil_div(a.n, POS);
  const unsigned slices = (unsigned)ceil_div(a.D, LPR * V);
  hipLaunchKernelGGL((embedding_grad_kernel<T, LPR, ROWS>), dim3((unsigned)blocks, slices), dim3(kEmbBlock), 0, stream,
                     a, g);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || blocks == 1) return e;
  hipLaunchKernelGGL((embedding_grad_join_kernel<V, LPR, ROWS>), dim3((unsigned)(blocks - 1), slices), dim3(kEmbBlock),
                     0, stream, a, g, POS);
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

hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, void* ws, hipStream_t stream) {
  const bool rows = a.unique_ids != nullptr || a.num_unique != nullptr;
  if (rows && a.n == 0) {
    hipLaunchKernelGGL(no_rows_kernel, dim3(1), dim3(1), 0, stream, a.num_unique);
    return hipGetLastError();
  }
  if (!rows && !a.accumulate) {
    const int64_t blocks = std::min(ceil_div(a.R * ceil_div(a.D, 4), kEmbBlock), kMaxGrid);
    hipLaunchKernelGGL(zero_rows_kernel, dim3((unsigned)blocks), dim3(kEmbBlock), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.n == 0) return hipSuccess;
  const GradLayout L = grad_layout(a.n, a.D);
  char* base = static_cast<char*>(ws);
  GradScratch g;
  g.pieces = reinterpret_cast<float*>(base + L.off_pieces);
  g.tail_run = reinterpret_cast<uint32_t*>(base + L.off_tail);
  if (rows) {
    const hipError_t e = launch_run_heads(a.keys, a.n, reinterpret_cast<uint32_t*>(base + L.off_tile),
                                          reinterpret_cast<uint32_t*>(base + L.off_group), &g.heads, stream);
    if (e != hipSuccess) return e;
    if (a.grad_type == GBA_F32) return grad_of<float, true>(a, g, stream);
    if (a.grad_type == GBA_BF16) return grad_of<bf16_t, true>(a, g, stream);
    return grad_of<f16_t, true>(a, g, stream);
  }
  if (a.grad_type == GBA_F32) return grad_of<float, false>(a, g, stream);
  if (a.grad_type == GBA_BF16) return grad_of<bf16_t, false>(a, g, stream);
  return grad_of<f16_t, false>(a, g, stream);
}

}  // namespace gba
