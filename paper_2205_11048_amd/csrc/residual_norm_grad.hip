// The gradient of a block's output joined to the residual stream (residual_norm.hip):
//   e = dh + pre'(dy),  dx = alpha e,  dz = post'(act(gate) e),
//   dgate = act'(gate) sum e u over the rows that share a gate row.
//
// Bound by bytes: 16,384 x 4096 bf16 with a gate for each 1024 rows 170 us (805 MB,
// 4.7 TB/s), 131,071 x 64 f32 with a gate for each row 63 (270 MB, 4.3); a second launch
// of 4 to 8 us joins the blocks' sums where there are several.  Four columns of a thread: with
// eight and twice the registers half as many waves wait for each other at two sums a
// row (264 us).  Rows of 4097 to 8192 columns take eight, spill, and read the weights
// again (8000 x 8192 bf16 270 us, 2.9 TB/s); wider ones are read three times (4000 x 16,384
// bf16 813).  Threads of a row go by powers of two: 32,548 x 1154 bf16 139 us (3.2 TB/s).
#include "residual_norm.hpp"

namespace gba {

constexpr int64_t kUnitBlocks = 512;        // most partial sums of the parameters' gradients
constexpr int kGradV = 4;                   // columns of a thread's vector

// How the rows are cut into units, the rows of a gate row (or all rows) in
// `cuts` equal parts: blocks take units in turn.
struct Units {
  uint32_t span;     // rows of a gate row whose gradients are added up; else all rows
  uint32_t cuts;     // units of it
  uint32_t rows;     // of a unit
  uint32_t units;
  uint32_t gates;    // rows of the gate
  bool shared;       // rows share the gate
  bool gate;         // ... and its gradient is asked for
  bool groups;       // a gate row for each group of lanes: units are as many gate rows as a block has groups
};
static Units units_of(const Args& a) {
  Units u;
  // (the same units, and so the same bits, with and without the gate's gradient)
  const bool shared = u.shared = a.gate_kind != GBA_GATE_NONE && a.gate_span > 1;
  u.gate = shared && a.dgate;
  const int64_t span = shared ? std::min(a.gate_span, a.n) : a.n, G = ceil_div(a.n, span);
  int64_t lanes = 1;   // no fewer rows to a unit than a block takes at a time
  while (lanes < kRegBlock && lanes * kGradV < a.D) lanes *= 2;
  const int64_t rows = std::max(ceil_div(span, std::max<int64_t>(1, kUnitBlocks / G)), std::min(span, kRegBlock / lanes));
  const int64_t cuts = ceil_div(span, rows);
  u.span = (uint32_t)span;
  u.gates = (uint32_t)G;
  // Few rows to a gate row, and many of these: side by side, not in turn by a block that has lanes for more rows
  // (239,128 x 32, bf16 beside a stream of f32, a gate for each ten rows 130 us -> 41; 200,000 x 128 bf16, one for each
  // four, 263 -> 70).  A block in turn takes gates / kUnitBlocks of them, a step each; side by side a step for each row.
  u.groups = shared && span < kRegBlock / lanes && G > kUnitBlocks * span;
  if (u.groups) {
    u.rows = u.span;
    u.cuts = 1;
    u.units = (uint32_t)ceil_div(G, kRegBlock / lanes);
    return u;
  }
  u.rows = (uint32_t)rows;
  u.cuts = (uint32_t)cuts;
  u.units = (uint32_t)(G * cuts);   // (below 2 n)
  return u;
}

// --------------------------------------------- rows read from memory again
// What the gradient of kV elements of a row is made of.
struct RowBack {
  float xh[kV], hh[kV];    // of the norm before: what was normalised, and dy by its weight
  float zh[kV], wz[kV];    // of the norm after the block, and its weight
  float u[kV];             // what the gate multiplies
  float f[kV], df[kV];     // the gate's factor and derivative
  float dy[kV], dh[kV];
};
struct RowStat {
  float mean_h, rstd_h, mean_z, rstd_z;
};
__device__ __forceinline__ RowStat row_stat(const Args& a, int64_t r) {
  RowStat s{0.0f, 1.0f, 0.0f, 1.0f};
  if (a.pre != GBA_ROW_NORM_NONE) s.rstd_h = a.pre_rstd[r];
  if (a.pre == GBA_ROW_NORM_LAYER) s.mean_h = a.pre_mean[r];
  if (a.post != GBA_ROW_NORM_NONE) s.rstd_z = a.post_rstd[r];
  if (a.post == GBA_ROW_NORM_LAYER) s.mean_z = a.post_mean[r];
  return s;
}
template <typename TS, typename TZ>
__device__ __forceinline__ void load_back(const Args& a, int64_t r, int c, const RowStat& s, bool after, RowBack& o) {
  const int count = a.D - c;
  float v[kV], w[kV], b[kV];
#pragma unroll
  for (int e = 0; e < kV; ++e) o.xh[e] = o.hh[e] = o.dy[e] = o.dh[e] = 0.0f;
  if (a.pre != GBA_ROW_NORM_NONE) {
    load_part<TS, kV>(static_cast<const TS*>(a.h) + r * a.h_stride + c, count, v);
    load_part<TZ, kV>(static_cast<const TZ*>(a.dy) + r * a.dy_stride + c, count, o.dy);
    load_param(a.pre_weight, a.weight_type, c, count, 1.0f, w);
#pragma unroll
    for (int e = 0; e < kV; ++e) {
      o.xh[e] = (v[e] - s.mean_h) * s.rstd_h;
      o.hh[e] = o.dy[e] * w[e];
    }
  }
  if (!after) return;
  if (a.dh) load_part<TS, kV>(static_cast<const TS*>(a.dh) + r * a.dh_stride + c, count, o.dh);
  load_part<TZ, kV>(static_cast<const TZ*>(a.z) + r * a.z_stride + c, count, v);
  load_param(a.post_weight, a.weight_type, c, count, 1.0f, o.wz);
  load_param(a.post_bias, a.weight_type, c, count, 0.0f, b);
  load_gate(a, r, c, count, o.f, o.df);
#pragma unroll
  for (int e = 0; e < kV; ++e) {
    o.zh[e] = (v[e] - s.mean_z) * s.rstd_z;
    o.u[e] = __builtin_fmaf(o.zh[e], o.wz[e], b[e]);
  }
}
// The gradient of h's element e: m1 and m2 are the means of hh (layer norm) and of hh * xh.
__device__ __forceinline__ float stream_grad(const RowBack& b, int e, const RowStat& s, float m1, float m2) {
  return b.dh[e] + s.rstd_h * (b.hh[e] - m1 - b.xh[e] * m2);
}

// A row's four means: of hh, of hh * xh, and the same of the norm after the block.
template <typename TS, typename TZ>
__global__ void __launch_bounds__(kRowBlock)
residual_norm_means_kernel(Args a, float* __restrict__ means) {
  __shared__ float s_sum[2][kRowWaves];
  const float D = (float)a.D;
  for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x) {
    const RowStat st = row_stat(a, r);
    float m[4] = {};
    RowBack b;
    if (a.pre != GBA_ROW_NORM_NONE) {
      for (int c = threadIdx.x * kV; c < a.D; c += kRowBlock * kV) {
        load_back<TS, TZ>(a, r, c, st, false, b);
#pragma unroll
        for (int e = 0; e < kV; ++e) {   // (past the row's end dy is 0)
          m[0] += b.hh[e];
          m[1] = __builtin_fmaf(b.hh[e], b.xh[e], m[1]);
        }
      }
      block_sum2(m[0], m[1], s_sum);
      m[0] = a.pre == GBA_ROW_NORM_LAYER ? m[0] / D : 0.0f;
      m[1] /= D;
    }
    if (a.post != GBA_ROW_NORM_NONE) {
      for (int c = threadIdx.x * kV; c < a.D; c += kRowBlock * kV) {
        load_back<TS, TZ>(a, r, c, st, true, b);
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          const float k = c + e < a.D ? stream_grad(b, e, st, m[0], m[1]) * b.f[e] * b.wz[e] : 0.0f;
          m[2] += k;
          m[3] = __builtin_fmaf(k, b.zh[e], m[3]);
        }
      }
      block_sum2(m[2], m[3], s_sum);
      m[2] = a.post == GBA_ROW_NORM_LAYER ? m[2] / D : 0.0f;
      m[3] /= D;
    }
    if (threadIdx.x < 4) means[r * 4 + threadIdx.x] = m[threadIdx.x];
  }
}

template <typename TS, typename TZ>
__global__ void __launch_bounds__(kRowBlock)
residual_norm_rows_kernel(Args a, const float* __restrict__ means) {
  const float alpha = (float)a.alpha;
  for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x) {
    const RowStat st = row_stat(a, r);
    float m[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) m[k] = means[r * 4 + k];
    for (int c = threadIdx.x * kV; c < a.D; c += kRowBlock * kV) {
      const int count = a.D - c;
      RowBack b;
      load_back<TS, TZ>(a, r, c, st, true, b);
      float dx[kV], dz[kV], dg[kV];
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const float g = stream_grad(b, e, st, m[0], m[1]);
        dx[e] = alpha * g;
        dg[e] = g * b.u[e] * b.df[e];
        const float k = g * b.f[e];
        dz[e] = a.post == GBA_ROW_NORM_NONE ? k : st.rstd_z * (k * b.wz[e] - m[2] - b.zh[e] * m[3]);
      }
      if (a.dx) store_part<TS, kV>(static_cast<TS*>(a.dx) + r * a.dx_stride + c, count, dx);
      if (a.dz) store_part<TZ, kV>(static_cast<TZ*>(a.dz) + r * a.dz_stride + c, count, dz);
      if (a.dgate && a.gate_span == 1) store_part<kV>(a.dgate, a.gate_type, r * a.dgate_stride + c, count, dg);
    }
  }
}

// Partial sums over units of rows: of the four parameters' gradients over all
// units of a block, of the gate's over each unit.  A wave per slice of
// columns, four waves' sums joined in LDS.
template <typename TS, typename TZ>
__global__ void __launch_bounds__(kRowBlock)
residual_norm_columns_kernel(Args a, const float* __restrict__ means, Units un, float* __restrict__ partial,
                             float* __restrict__ gate_partial) {
  __shared__ float s_part[kRowWaves][kWave * kV];
  const int w = threadIdx.x / kWave, lane = lane_id();
  const int c = (int)blockIdx.y * (kWave * kV) + lane * kV;
  float sum[4][kV] = {};
  // adds up `v` over the waves and hands each column's sum to `to`
  auto join = [&](float (&v)[kV], auto to) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kV; ++e) s_part[w][lane * kV + e] = v[e];
    __syncthreads();
    const int64_t cc = (int64_t)blockIdx.y * (kWave * kV) + threadIdx.x;
    float t = 0.0f;
#pragma unroll
    for (int k = 0; k < kRowWaves; ++k) t += s_part[k][threadIdx.x];
    if (cc < a.D) to(cc, t);
  };
  static_assert(kRowBlock == kWave * kV, "a thread per column of the slice");
  for (int64_t u = blockIdx.x; u < (int64_t)un.units; u += gridDim.x) {
    const int64_t g = (uint32_t)u / un.cuts, first = g * un.span + ((uint32_t)u - g * un.cuts) * un.rows;
    int64_t end = first + un.rows;
    end = end < (g + 1) * (int64_t)un.span ? end : (g + 1) * (int64_t)un.span;
    end = end < a.n ? end : a.n;
    float dg[kV] = {};
    if (c < a.D) {
      for (int64_t r = first + w; r < end; r += kRowWaves) {
        const RowStat st = row_stat(a, r);
        RowBack b;
        load_back<TS, TZ>(a, r, c, st, true, b);
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          const float gr = stream_grad(b, e, st, means[r * 4], means[r * 4 + 1]);
          dg[e] += gr * b.u[e] * b.df[e];
          const float k = gr * b.f[e];
          sum[0][e] = __builtin_fmaf(k, b.zh[e], sum[0][e]);
          sum[1][e] += k;
          sum[2][e] = __builtin_fmaf(b.dy[e], b.xh[e], sum[2][e]);
          sum[3][e] += b.dy[e];
        }
      }
    }
    if (un.gate)
      join(dg, [&](int64_t cc, float t) {
        const float v[1] = {t};
        if (un.cuts == 1) store_part<1>(a.dgate, a.gate_type, g * a.dgate_stride + cc, 1, v);
        else gate_partial[u * a.D + cc] = t;
      });
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    join(sum[k], [&](int64_t cc, float t) { partial[((int64_t)blockIdx.x * 4 + k) * a.D + cc] = t; });
}

// ------------------------------------------------------ rows in registers
// Where a block is in its units: at rows rb .. of unit u, whose last is end - 1.
struct UnitCursor {
  uint32_t u, g, rb, end;
  __device__ __forceinline__ void enter(const Units& un, uint32_t n) {
    g = u / un.cuts;
    rb = g * un.span + (u - g * un.cuts) * un.rows;
    end = min(min(rb + un.rows, (g + 1) * un.span), n);
  }
};

// The kernel's arguments, read again: what is needed where a unit or the kernel
// ends would otherwise stay in scalar registers over all rows, which have no room
// for it (a wave kept 70 of them in lanes of vector registers).
typedef const __attribute__((address_space(4))) Args* LateArgs;
__device__ __forceinline__ LateArgs late_args() {
  LateArgs p = (LateArgs)__builtin_amdgcn_kernarg_segment_ptr();   // (the first argument)
  asm volatile("" : "+s"(p));
  return p;
}

// How the gate goes by rows: a row each (or no gate), a unit of rows that share
// one for each block, units in turn, or a gate row for each group of lanes, which
// takes its rows one after another.
enum GateRows { kGateEach, kGateUnit, kGateUnits, kGateGroups };

// A sigmoid gate's factor f and its derivative f (1 - f) from one number, the smaller of f and 1 - f, which has all
// its digits; 1 - f with its sign turned round.  (8192 x 4096 bf16, a gate for each row: 140 us, and 158 with the gate
// read again for its derivative; f and 1 - f both in registers spill in units of rows.)
__device__ __forceinline__ float gate_code(float a) {
  float f, i;
  sigmoid_both(a, f, i);
  return a < 0.0f ? f : -i;
}
__device__ __forceinline__ float gate_factor(int kind, float code) {
  return kind == GBA_GATE_SIGMOID && (__float_as_uint(code) >> 31) ? 1.0f + code : code;
}
__device__ __forceinline__ float gate_derivative(int kind, float code) {
  const float least = fabsf(code);
  return kind == GBA_GATE_SIGMOID ? least * (1.0f - least) : 1.0f;
}

// A thread keeps its columns of the parameters' sums and of the weights in
// registers from row to row.  Foreign columns (RowPlace) have weights of 0, so
// that they add nothing to the row's sums, and are neither stored nor joined; a
// row past the unit's end is the last one again with gradients of 0.  A row's
// arrays are loaded again as soon as the row before it has taken them.
// Of the rows that share a gate the sums of e zh and e are enough: the gate and
// post's parameters take from these what they need when the unit ends.
template <typename TS, typename TZ, int LPR, int NV, GateRows ROWS>
__global__ void __launch_bounds__((NormShape<kGradV, LPR, NV>::BLOCK), 4)
residual_norm_grad_kernel(Args a, Units un, float* __restrict__ partial, float* __restrict__ gate_partial) {
  typedef NormShape<kGradV, LPR, NV> S;
  constexpr int V = S::V;
  constexpr int TEAM = LPR < kWave ? kWave : LPR;
  constexpr int TEAMS = S::BLOCK / TEAM;
  constexpr int COLS = LPR * S::E;
  typedef typename VecOf<TS, V>::type stream_vec;
  typedef typename VecOf<TZ, V>::type vec;
  __shared__ float s_sum[2][2][S::WAVES];
  __shared__ float s_part[TEAMS > 1 ? TEAMS * COLS : 1];
  const uint32_t gl = threadIdx.x % LPR, grp = S::G == 1 ? 0 : threadIdx.x / LPR;   // (a row's addresses are then uniform)
  const RowPlace<V, LPR, NV, false> at(gl, a.D);
  const float inv_D = 1.0f / (float)a.D, alpha = (float)a.alpha;
  const bool pre = a.pre != GBA_ROW_NORM_NONE, post = a.post != GBA_ROW_NORM_NONE;
  const bool each = ROWS == kGateEach && a.gate_kind != GBA_GATE_NONE;
  // post's weight and bias, pre's; units in turn: of the rows' sums of e zh and e, whose place is else the first two's
  constexpr bool GROUPS = ROWS == kGateGroups;
  constexpr int SUMS = ROWS == kGateUnits || GROUPS ? 6 : 4, W = SUMS == 6 ? 4 : 0;
  // f: the gate's codes, or the factors, with the codes made once more where a unit ends (8000 x 8192, a sigmoid gate for
  // each 1000 rows: bf16 300 us with codes and 271 with factors, beside a stream of f32 414 and 410, all f32 491 and 564)
  constexpr bool CODES = ROWS == kGateEach || NV == 1 || sizeof(TZ) == 4;
  constexpr bool KEEP = NV == 1;   // the weights (two vectors of a thread leave no registers for them)
  float wz[NV][V], wh[NV][V], f[NV][V], sum[SUMS][NV][V];
  auto weights = [&](const void* p, int type, float (&w)[NV][V]) {
    load_params(at, p, type, 1.0f, w);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) w[k][e] = at.own(k, e) ? w[k][e] : 0.0f;
  };
  if constexpr (KEEP) {
    weights(a.post_weight, a.weight_type, wz);
    weights(a.pre_weight, a.weight_type, wh);
  }
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      f[k][e] = 1.0f;
#pragma unroll
      for (int i = 0; i < SUMS; ++i) sum[i][k][e] = 0.0f;
    }
  stream_vec h[NV] = {}, dh[NV] = {};
  vec z[NV] = {}, dy[NV] = {};
  RowStat st, stn;
  const uint32_t n = (uint32_t)a.n;
  auto place_of = [&](const UnitCursor& c) { return GROUPS ? (c.g + grp) * un.span + c.rb : c.rb + grp; };
  auto row_of = [&](const UnitCursor& c) { return (int64_t)min(place_of(c), (GROUPS ? n : c.end) - 1); };
  auto load_pre = [&](int64_t r) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      h[k] = at.load_raw(static_cast<const TS*>(a.h) + r * a.h_stride, k);
      dy[k] = at.load_raw(static_cast<const TZ*>(a.dy) + r * a.dy_stride, k);
    }
  };
  auto load_post = [&](int64_t r) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      z[k] = at.load_raw(static_cast<const TZ*>(a.z) + r * a.z_stride, k);
      if (a.dh) dh[k] = at.load_raw(static_cast<const TS*>(a.dh) + r * a.dh_stride, k);
    }
  };
  // adds `v` up over the block's rows and hands each column's sum to `to`
  auto join = [&](float (&v)[NV][V], auto to) {
    if constexpr (LPR < kWave) {
#pragma unroll
      for (int off = LPR; off < kWave; off <<= 1)
#pragma unroll
        for (int e = 0; e < V; ++e) v[0][e] += __shfl_xor(v[0][e], off, kWave);   // (NV is 1)
    }
    if constexpr (TEAMS > 1) {
      __syncthreads();   // the last sums have been read
      if ((int)(threadIdx.x % TEAM) < LPR) {
        float* s = s_part + threadIdx.x / TEAM * COLS;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (at.own(k, e)) s[at.col[k] + e] = v[k][e];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < a.D; c += S::BLOCK) {
        float t = 0.0f;
#pragma unroll
        for (int m = 0; m < TEAMS; ++m) t += s_part[m * COLS + c];
        to(c, t);
      }
    } else {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (at.own(k, e)) to(at.col[k] + e, v[k][e]);
    }
  };
  // (GROUPS: g is the first group's gate row, and rb .. end - 1 are places in the gate rows)
  auto enter = [&](UnitCursor& c) {
    if constexpr (GROUPS) {
      c.g = c.u * S::G;
      c.rb = 0;
      c.end = un.span;
    } else {
      c.enter(un, n);
    }
  };
  UnitCursor now{blockIdx.x, 0, 0, 0};
  enter(now);
  {
    const int64_t r = row_of(now);
    st = row_stat(a, r);
    if (pre) load_pre(r);
    load_post(r);
  }
  bool entered = true;
  int buffer = 0;
  for (;;) {
    UnitCursor next = now;
    next.rb += GROUPS ? 1 : S::G;
    const bool leaves = next.rb >= now.end;
    if (leaves) {
      next.u += gridDim.x;
      if (next.u < un.units) enter(next);
    }
    const bool more = next.u < un.units;
    const int64_t r = place_of(now), next_row = more ? row_of(next) : 0;
    const bool active = place_of(now) < (GROUPS ? n : now.end);   // (the last gate row's units may have no rows)
    auto load_gate_codes = [&](LateArgs l) {
      load_gate_row(at, l->gate, l->gate_type, (each ? r : (int64_t)(GROUPS ? min(now.g + grp, un.gates - 1) : now.g)) * l->gate_stride, f);
      if (l->gate_kind != GBA_GATE_SIGMOID) return;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) f[k][e] = gate_code(f[k][e]);
    };
    auto factors_of_codes = [&](int kind) {
      if constexpr (!CODES) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e) f[k][e] = gate_factor(kind, f[k][e]);
      }
    };
    auto factor = [&](int k, int e) { return CODES ? gate_factor(a.gate_kind, f[k][e]) : f[k][e]; };
    if (each ? active : ROWS != kGateEach && entered) {
      const LateArgs l = late_args();
      load_gate_codes(l);
      factors_of_codes(l->gate_kind);
    }
    if (!active) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        dy[k] = vec{};
        dh[k] = stream_vec{};
      }
    }
    // the stream's gradient
    float e_[NV][V], t[2] = {0.0f, 0.0f};
    if (pre) {
      if constexpr (!KEEP) {
        const LateArgs l = late_args();
        weights(l->pre_weight, l->weight_type, wh);
      }
      float xh[NV][V];
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float g = (float)dy[k][e];
          xh[k][e] = ((float)h[k][e] - st.mean_h) * st.rstd_h;
          e_[k][e] = g * wh[k][e];
          t[0] += e_[k][e];
          t[1] = __builtin_fmaf(e_[k][e], xh[k][e], t[1]);
          sum[2][k][e] = __builtin_fmaf(g, xh[k][e], sum[2][k][e]);
          sum[3][k][e] += g;
        }
      if (more) load_pre(next_row);
      row_total<LPR, S::WAVES>(t, s_sum, buffer);
      const float m1 = a.pre == GBA_ROW_NORM_LAYER ? t[0] * inv_D : 0.0f, m2 = t[1] * inv_D;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e)
          e_[k][e] = __builtin_fmaf(st.rstd_h, __builtin_fmaf(-xh[k][e], m2, e_[k][e] - m1), (float)dh[k][e]);
    } else {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) e_[k][e] = (float)dh[k][e];
    }
    // the block's
    if constexpr (!KEEP) {
      const LateArgs l = late_args();
      weights(l->post_weight, l->weight_type, wz);
    }
    float zh[NV][V], kk[NV][V];
    t[0] = t[1] = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        zh[k][e] = ((float)z[k][e] - st.mean_z) * st.rstd_z;
        const float g = e_[k][e] * factor(k, e), s = ROWS == kGateEach ? g : e_[k][e];
        sum[W][k][e] = __builtin_fmaf(s, zh[k][e], sum[W][k][e]);
        sum[W + 1][k][e] += s;
        kk[k][e] = g * wz[k][e];
        t[0] += kk[k][e];
        t[1] = __builtin_fmaf(kk[k][e], zh[k][e], t[1]);
        if (!post) kk[k][e] = g;
      }
    if (each && a.dgate && active) {
      const LateArgs l = late_args();
      float bz[NV][V];
      load_params(at, l->post_bias, l->weight_type, 0.0f, bz);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float u = __builtin_fmaf(zh[k][e], wz[k][e], bz[k][e]);
          o[e] = e_[k][e] * u * gate_derivative(l->gate_kind, f[k][e]);
        }
        const int64_t to = r * l->dgate_stride;
        if (l->gate_type == GBA_F32) at.store_own(static_cast<float*>(l->dgate) + to, k, o);
        else if (l->gate_type == GBA_BF16) at.store_own(static_cast<bf16_t*>(l->dgate) + to, k, o);
        else at.store_own(static_cast<f16_t*>(l->dgate) + to, k, o);
      }
    }
    if (more) {
      stn = row_stat(a, next_row);
      load_post(next_row);
    }
    if (post) {
      row_total<LPR, S::WAVES>(t, s_sum, buffer);
      const float m1 = a.post == GBA_ROW_NORM_LAYER ? t[0] * inv_D : 0.0f, m2 = t[1] * inv_D;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) kk[k][e] = st.rstd_z * __builtin_fmaf(-zh[k][e], m2, kk[k][e] - m1);
    } else if (LPR > kWave && !pre) {
      __syncthreads();   // dx may be dh, dz dy: all of the row has been read
    }
    if (active) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = alpha * e_[k][e];
        if (a.dx) at.store_own(static_cast<TS*>(a.dx) + r * a.dx_stride, k, o);
        if (a.dz) at.store_own(static_cast<TZ*>(a.dz) + r * a.dz_stride, k, kk[k]);
      }
    }
    if (ROWS != kGateEach && leaves) {
      if (un.gate) {
        const LateArgs l = late_args();
        float dg[NV][V];
        load_params(at, l->post_bias, l->weight_type, 0.0f, dg);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e) dg[k][e] = __builtin_fmaf(wz[k][e], sum[W][k][e], dg[k][e] * sum[W + 1][k][e]);
        if constexpr (!CODES) load_gate_codes(late_args());
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e) dg[k][e] *= gate_derivative(l->gate_kind, f[k][e]);
        factors_of_codes(l->gate_kind);
        if constexpr (GROUPS) {
          const int64_t to = (int64_t)(now.g + grp) * l->dgate_stride;
          if (now.g + grp < un.gates) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
              if (l->gate_type == GBA_F32) at.store_own(static_cast<float*>(l->dgate) + to, k, dg[k]);
              else if (l->gate_type == GBA_BF16) at.store_own(static_cast<bf16_t*>(l->dgate) + to, k, dg[k]);
              else at.store_own(static_cast<f16_t*>(l->dgate) + to, k, dg[k]);
            }
          }
        } else {
          join(dg, [&](int c, float v) {
            const float o[1] = {v};
            if (un.cuts == 1) store_part<1>(l->dgate, l->gate_type, now.g * l->dgate_stride + c, 1, o);
            else gate_partial[(int64_t)now.u * a.D + c] = v;
          });
        }
      }
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if constexpr (SUMS == 6) {
            sum[0][k][e] = __builtin_fmaf(factor(k, e), sum[W][k][e], sum[0][k][e]);
            sum[1][k][e] = __builtin_fmaf(factor(k, e), sum[W + 1][k][e], sum[1][k][e]);
            sum[W][k][e] = sum[W + 1][k][e] = 0.0f;
          } else {
            sum[0][k][e] *= factor(k, e);
            sum[1][k][e] *= factor(k, e);
          }
        }
    }
    if (!more) break;
    now = next;
    entered = leaves;
    st = stn;
  }
  const LateArgs l = late_args();
  void* const outs[4] = {l->dpost_weight, l->dpost_bias, l->dpre_weight, l->dpre_bias};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (!outs[i]) continue;
    join(sum[i], [&](int c, float v) {
      const float o[1] = {v};
      if (gridDim.x == 1) store_part<1>(outs[i], l->grad_type, c, 1, o);   // the only block writes the sums themselves
      else partial[((int64_t)blockIdx.x * 4 + i) * a.D + c] = v;
    });
  }
}

// The parameters' gradients from the blocks' partial sums, and the gate's from
// the units': 64 columns a block, each wave a share of the sums.
constexpr int kJoinBlock = 1024;
constexpr int kJoinWaves = kJoinBlock / kWave;
__global__ void __launch_bounds__(kJoinBlock)
residual_norm_join_kernel(Args a, const float* __restrict__ partial, int64_t parts, Units un,
                          const float* __restrict__ gate_partial) {
  __shared__ float s_sum[kJoinWaves][kWave];
  const int w = threadIdx.x / kWave, lane = lane_id();
  const int64_t c = (int64_t)blockIdx.x * kWave + lane;
  const int which = (int)blockIdx.y;   // a parameter, or 4 + a gate row
  void* const out = which == 0 ? a.dpost_weight : which == 1 ? a.dpost_bias : which == 2 ? a.dpre_weight : a.dpre_bias;
  if (which < 4 && !out) return;
  const float* from = which < 4 ? partial + which * (int64_t)a.D : gate_partial + (int64_t)(which - 4) * un.cuts * a.D;
  const int64_t count = which < 4 ? parts : un.cuts, step = which < 4 ? 4 * (int64_t)a.D : a.D;
  float s[1] = {0.0f};
  if (c < a.D) {
#pragma unroll 8
    for (int64_t p = w; p < count; p += kJoinWaves) s[0] += from[p * step + c];
  }
  s_sum[w][lane] = s[0];
  __syncthreads();
  if (w != 0 || c >= a.D) return;
  s[0] = 0.0f;
#pragma unroll
  for (int k = 0; k < kJoinWaves; ++k) s[0] += s_sum[k][lane];
  if (which >= 4) {
    store_part<1>(a.dgate, a.gate_type, (which - 4) * a.dgate_stride + c, 1, s);
    return;
  }
  store_part<1>(out, a.grad_type, c, 1, s);
}

// ------------------------------------------------------------- launching
// Scratch: partial sums of the parameters' gradients (a row of four per block)
// and of the gate's (a row per unit), and a row's means.
struct NormRoom {
  size_t partial, gate, means, bytes;
};
static NormRoom norm_room(int64_t n, int32_t D) {
  NormRoom r;
  // (units: at most as many as rows of whole gate rows, below 2 n; fewer than 2 kUnitBlocks where they are joined)
  r.partial = 0;
  r.gate = align_up((size_t)std::min(2 * n, kUnitBlocks) * 4 * D * sizeof(float));
  r.means = r.gate + align_up((size_t)std::min(2 * n, 2 * kUnitBlocks) * D * sizeof(float));
  r.bytes = r.means + align_up((size_t)n * 4 * sizeof(float)) + 256;
  return r;
}
size_t residual_norm_grad_workspace_bytes(int64_t n, int32_t D) { return norm_room(n, D).bytes; }

// Calls f.run<LPR, NV>() for the shape of rows of D columns: a vector of a
// thread up to the widest block, two beyond.
template <int LPR, typename F>
static hipError_t with_grad_shape(int32_t D, const F& f) {
  if (D <= LPR * kGradV) return f.template run<LPR, 1>();
  if constexpr (LPR < kWidest) return with_grad_shape<2 * LPR>(D, f);
  else return f.template run<LPR, 2>();
}

template <typename TS, typename TZ>
struct RowsBackward {
  const Args& a;
  const Units& un;
  float* partial;
  float* gate;
  hipStream_t stream;
  template <int LPR, int NV, GateRows ROWS>
  void launch(unsigned grid) const {
    hipLaunchKernelGGL((residual_norm_grad_kernel<TS, TZ, LPR, NV, ROWS>), dim3(grid), dim3(NormShape<kGradV, LPR, NV>::BLOCK),
                       0, stream, a, un, partial, gate);
  }
  template <int LPR, int NV>
  void launch_groups(unsigned grid) const {
    if constexpr (NormShape<kGradV, LPR, NV>::G > 1) launch<LPR, NV, kGateGroups>(grid);
  }
  template <int LPR, int NV>
  hipError_t run() const {
    const unsigned grid = (unsigned)std::min<int64_t>(un.units, kUnitBlocks);
    if (!un.shared) launch<LPR, NV, kGateEach>(grid);
    else if (un.groups) launch_groups<LPR, NV>(grid);
    else if ((int64_t)un.units <= kUnitBlocks) launch<LPR, NV, kGateUnit>(grid);
    else launch<LPR, NV, kGateUnits>(grid);
    return hipGetLastError();
  }
};

template <typename TS, typename TZ>
static hipError_t backward_as(const Args& a, void* ws, hipStream_t stream) {
  const NormRoom room = norm_room(a.n, a.D);
  float* partial = reinterpret_cast<float*>(static_cast<char*>(ws) + room.partial);
  float* gate = reinterpret_cast<float*>(static_cast<char*>(ws) + room.gate);
  float* means = reinterpret_cast<float*>(static_cast<char*>(ws) + room.means);
  const Units un = units_of(a);
  const bool params = a.dpost_weight || a.dpost_bias || a.dpre_weight || a.dpre_bias;
  const int64_t parts = std::min<int64_t>(un.units, kUnitBlocks);
  if (a.D <= kRegColumns) {
    const hipError_t e = with_grad_shape<1>(a.D, RowsBackward<TS, TZ>{a, un, partial, gate, stream});
    if (e != hipSuccess) return e;
  } else {
    const unsigned rows = (unsigned)std::min(a.n, kMaxRowGrid);
    hipLaunchKernelGGL((residual_norm_means_kernel<TS, TZ>), dim3(rows), dim3(kRowBlock), 0, stream, a, means);
    // (the columns before the rows: dx may take dh's place, and dz dy's)
    if (params || un.gate) {
      const dim3 grid((unsigned)parts, (unsigned)ceil_div(a.D, kWave * kV));
      hipLaunchKernelGGL((residual_norm_columns_kernel<TS, TZ>), grid, dim3(kRowBlock), 0, stream, a,
                         (const float*)means, un, partial, gate);
    }
    if (a.dx || a.dz || (a.dgate && a.gate_span == 1))
      hipLaunchKernelGGL((residual_norm_rows_kernel<TS, TZ>), dim3(rows), dim3(kRowBlock), 0, stream, a,
                         (const float*)means);
  }
  const int64_t joined = un.gate && un.cuts > 1 ? un.units / un.cuts : 0;
  if ((params && !(parts == 1 && a.D <= kRegColumns)) || joined)
    hipLaunchKernelGGL(residual_norm_join_kernel, dim3((unsigned)ceil_div(a.D, kWave), (unsigned)(4 + joined)),
                       dim3(kJoinBlock), 0, stream, a, (const float*)partial, parts, un, (const float*)gate);
  return hipGetLastError();
}

struct Backward {
  const Args& a;
  void* ws;
  hipStream_t stream;
  template <typename TS, typename TZ>
  hipError_t run() const { return backward_as<TS, TZ>(a, ws, stream); }
};

static __global__ void __launch_bounds__(kRowBlock) residual_norm_zero_kernel(Args a) {
  const float none[1] = {0.0f};
  const int64_t c = (int64_t)blockIdx.x * kRowBlock + threadIdx.x;
  if (c >= a.D) return;
  if (a.dpost_weight) store_part<1>(a.dpost_weight, a.grad_type, c, 1, none);
  if (a.dpost_bias) store_part<1>(a.dpost_bias, a.grad_type, c, 1, none);
  if (a.dpre_weight) store_part<1>(a.dpre_weight, a.grad_type, c, 1, none);
  if (a.dpre_bias) store_part<1>(a.dpre_bias, a.grad_type, c, 1, none);
}

hipError_t launch_residual_norm_grad(const Args& a, void* ws, hipStream_t stream) {
  if (a.n > 0) return with_types(a, Backward{a, ws, stream});
  hipLaunchKernelGGL(residual_norm_zero_kernel, dim3((unsigned)ceil_div(a.D, kRowBlock)), dim3(kRowBlock), 0, stream, a);
  return hipGetLastError();
}

}  // namespace gba
