// Selective state space scan and its gradient (include/lsgd.h): the kernels of one activation type.
//
//   h_t = exp(delta_t A) h_(t-1) + delta_t x_t B_t,   y_t = C_t . h_t
//
// for N states of every channel.  A block takes 256 / L channels of a run of rows (a chain); L lanes share a channel and hold 4 states
// each in registers, so N <= 4 L.  Rows are staged in shared memory a tile at a time as what the recurrence reads: delta
// and delta x (one softplus a row and channel), B and C as fp32.  The sums over a channel's states go through L lanes, four rows at
// once (each lane ends up with one row's sum), and are finished (skip, gate) by the thread that staged the row's piece.
//
// Chains.  Where workers, sequences and channels give enough blocks, a chain is a run of whole sequences and nothing else is
// needed.  Otherwise the rows are split into chains of equal length: a first pass finds what every chain adds to the state behind
// it and by how much it decays the state in front (one exp of the summed time steps), a short pass runs over the chains, and
// the last pass starts every chain from its own state.  The exps are then computed twice.
//
// Gradient.  The forward pass saves the state in front of every 8th row.  A chain goes backwards in groups of 8 rows: it recomputes
// the group's states from the saved one, keeps them and the decays in registers, and runs the adjoint
//   g_t = d_t C_t + a_(t+1) g_(t+1)
// back through them.  dB and dC are sums over channels: over the warp's by exchanges that halve the number of values at each step,
// over the warps in shared memory, over the blocks by a second kernel; all in a fixed order.
#pragma once
#include "seq.h"

namespace lsgd {
namespace scan {

constexpr int kThreads = 256, kQuad = 4, kGroup = 8;
template <int L> struct Tile {
  static constexpr int kCh = kThreads / L;               // channels of a block
  static constexpr int kRows = L == 2 ? 16 : 32;         // rows of a tile: at most one piece of 8 channels a thread
  static constexpr int kN = kQuad * L;                   // states, padded
  static constexpr int kPieces = kCh / 8 * kRows;
};
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Args {
  lsgd_scan_desc d;
  SeqView q;
  int32_t chains, per;       // chains of a worker; sequences of a chain, or (split) rows
  int32_t split, wide;       // wide: every row can be moved 8 values at a time
  uint32_t tiles;            // blocks of channels
  float* ends;               // split: [P][chains][D][N], what a chain adds, then the state (adjoint) it starts from
  float* sums;               // split: [P][chains][D], summed time steps; negative where a sequence begins inside
  float* old_state;          // split, with a state: its copy, [P][S][D][N]
  float* part_bc;            // backward: [P][tiles][T][2][N]
  float* part_a;             // backward: [P][chains][D][N]
  float* part_v;             // backward: [P][chains][2][D]
};

template <typename T>
__device__ __forceinline__ Rows<T> view(const lsgd_rows& r) {
  return Rows<T>{static_cast<T*>(r.data), r.ld, r.stride};
}
__device__ __forceinline__ float ex2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// softplus(v) = max(v, 0) + log1p(e), e = exp(-|v|) <= 1; log1p(e) = 2 artanh(e / (2 + e)) by its series (s <= 1/3).
__device__ __forceinline__ float softplus(float v, float& e) {
  e = expf(-fabsf(v));
  const float s = __fdividef(e, 2.f + e), s2 = s * s;
  float r = fmaf(s2, 1.f / 13, 1.f / 11);
  r = fmaf(s2, r, 1.f / 9);
  r = fmaf(s2, r, 1.f / 7);
  r = fmaf(s2, r, 1.f / 5);
  r = fmaf(s2, r, 1.f / 3);
  return fmaxf(v, 0.f) + 2.f * fmaf(s * s2, r, s);
}
__device__ __forceinline__ float sigmoid(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }

// 8 neighbouring channels of a row; those behind the last are zeros.
template <typename T>
__device__ __forceinline__ void load8(Pack<T, 8>& k, const T* row, int ch, int D, bool wide) {
  if (wide) {
    k.load(row + ch);
    return;
  }
  float f[8];
#pragma unroll
  for (int v = 0; v < 8; ++v) {
    Pack<T, 1> one;
    f[v] = 0.f;
    if (ch + v < D) {
      one.load(row + ch + v);
      one.get(f + v);
    }
  }
  k.set(f);
}
template <typename T>
__device__ __forceinline__ void store8(const float (&f)[8], T* row, int ch, int D, bool wide) {
  if (wide) {
    Pack<T, 8> k;
    k.set(f);
    k.store(row + ch);
    return;
  }
#pragma unroll
  for (int v = 0; v < 8; ++v)
    if (ch + v < D) {
      Pack<T, 1> one;
      one.set(f + v);
      one.store(row + ch + v);
    }
}

// A thread's place: its channel and states in the recurrence.
template <int L>
struct Place {
  int local, ch, n0;         // channel in the block and in the row, first of 4 states
  bool in;
  __device__ __forceinline__ Place(uint32_t tile, int D) {
    local = threadIdx.x / L;
    ch = tile * Tile<L>::kCh + local;
    n0 = (threadIdx.x % L) * kQuad;
    in = ch < D;
  }
};

// A log2(e) of the thread's states; 0 for those that do not exist (they stay zero, for B is zero there)
template <int L>
__device__ __forceinline__ void decay_rates(const Args& a, int p, const Place<L>& at, float (&A2)[kQuad]) {
#pragma unroll
  for (int k = 0; k < kQuad; ++k) {
    A2[k] = 0.f;
    if (at.in && at.n0 + k < a.d.N)
      A2[k] = -expf(static_cast<const float*>(a.d.a_log.data)[p * a.d.a_log.stride + at.ch * a.d.a_log.ld + at.n0 + k]) * kLog2e;
  }
}

// 4 states of a channel in a [..][D][N] array of fp32, whose row `row` is (.., channel)
__device__ __forceinline__ void load_states(const float* base, int64_t row, int n0, int N, float (&h)[kQuad]) {
  const float* src = base + row * N + n0;
  if ((N & 3) == 0) {
    const float4 v = *reinterpret_cast<const float4*>(src);
    h[0] = v.x, h[1] = v.y, h[2] = v.z, h[3] = v.w;
  } else {
#pragma unroll
    for (int k = 0; k < kQuad; ++k) h[k] = n0 + k < N ? src[k] : 0.f;
  }
}
__device__ __forceinline__ void store_states(float* base, int64_t row, int n0, int N, const float (&h)[kQuad]) {
  float* dst = base + row * N + n0;
  if ((N & 3) == 0) {
    *reinterpret_cast<float4*>(dst) = make_float4(h[0], h[1], h[2], h[3]);
  } else {
#pragma unroll
    for (int k = 0; k < kQuad; ++k)
      if (n0 + k < N) dst[k] = h[k];
  }
}
// whether the thread's 4 states exist as a whole or in part
template <int L>
__device__ __forceinline__ bool has_states(const Place<L>& at, int N) { return at.in && at.n0 < N; }

struct Range {
  int t0, t1, base;          // rows of the chain; base: t0 rounded down to a group
  __device__ __forceinline__ Range(const Args& a, int p, int c) {
    if (a.split) {
      t0 = min(a.q.T, c * a.per);
      t1 = min(a.q.T, t0 + a.per);
    } else {
      const int s0 = c * a.per, s1 = min(a.q.S, s0 + a.per);
      t0 = a.q.edge(p, s0);
      t1 = a.q.edge(p, s1);
    }
    base = t0 & ~(kGroup - 1);
  }
};

// Sums over the L lanes of a channel for four rows.  L >= 4: lane l holds row row_of(l) in y[0]; L == 2: rows 2 (l & 1) and one more.
template <int L>
__device__ __forceinline__ void sum_states(float (&y)[4], int lane) {
  const bool b0 = lane & 1;
  const float s0 = b0 ? y[0] : y[2], s1 = b0 ? y[1] : y[3];
  y[0] = (b0 ? y[2] : y[0]) + __shfl_xor_sync(0xFFFFFFFFu, s0, 1);
  y[1] = (b0 ? y[3] : y[1]) + __shfl_xor_sync(0xFFFFFFFFu, s1, 1);
  if (L == 2) return;
  const bool b1 = lane & 2;
  const float s = b1 ? y[0] : y[1];
  y[0] = (b1 ? y[1] : y[0]) + __shfl_xor_sync(0xFFFFFFFFu, s, 2);
#pragma unroll
  for (int m = 4; m < L; m *= 2) y[0] += __shfl_xor_sync(0xFFFFFFFFu, y[0], m);
}
__device__ __forceinline__ int row_of(int lane) { return 2 * (lane & 1) + ((lane >> 1) & 1); }

// Which rows of a tile begin and end a sequence (its number, else -1), and whether a row belongs to the chain.
template <int L>
__device__ __forceinline__ bool mark_rows(const Args& a, int p, const Range& r, int base, int* begins, int* ends) {
  bool special = false;
  const int i = threadIdx.x;
  if (i < Tile<L>::kRows) {
    const int t = base + i;
    int b = -1, e = -1;
    if (t >= r.t0 && t < r.t1) {
      const int code = a.q.code(p, t);
      if (code >= 0) {
        if (a.q.code(p, t - 1) != code) b = code;
        if (a.q.code(p, t + 1) != code) e = code;
      }
    }
    begins[i] = b;
    ends[i] = e;
    special = b >= 0 || e >= 0;
  }
  return special;
}
__device__ __forceinline__ bool row_lives(const Args& a, int p, const Range& r, int t) {
  return t >= r.t0 && t < r.t1 && (!a.q.starts || a.q.code(p, t) >= 0);
}

template <typename T, int L>
__device__ __forceinline__ void stage_bc(const Args& a, int p, const Range& r, int base, const lsgd_rows& src, float* dst) {
  constexpr int N = Tile<L>::kN;
  const Rows<T> v = view<T>(src);
  for (int i = threadIdx.x; i < Tile<L>::kRows * N; i += kThreads) {
    const int t = base + i / N, n = i % N;
    float f = 0.f;
    if (n < a.d.N && row_lives(a, p, r, t)) {
      Pack<T, 1> one;
      one.load(v.row(p, t) + n);
      one.get(&f);
    }
    dst[i] = f;
  }
}

// ------------------------------------------------------------------------------------------------ forward
// kEnds: only what the chain adds to the state behind it, and its summed time steps.
template <typename T, int L, bool kEnds>
__global__ void __launch_bounds__(kThreads, 3) forward_kernel(const __grid_constant__ Args a) {
  using Ti = Tile<L>;
  pdl_wait();
  pdl_launch_dependents();
  __shared__ __align__(16) float2 s_dd[Ti::kRows * Ti::kCh];       // delta, delta x; then the sum over the states
  __shared__ __align__(16) float s_b[Ti::kRows * Ti::kN], s_c[kEnds ? 4 : Ti::kRows * Ti::kN];
  __shared__ int s_begin[Ti::kRows], s_end[Ti::kRows];
  const int p = blockIdx.z, c = blockIdx.y, lane = threadIdx.x & 31;
  const Range r(a, p, c);
  const lsgd_scan_desc& d = a.d;
  const Place<L> at(blockIdx.x, d.D);
  const bool mine = has_states<L>(at, d.N);
  const int64_t chain_row = ((int64_t)p * a.chains + c) * d.D + at.ch;
  float A2[kQuad], h[kQuad] = {};
  decay_rates<L>(a, p, at, A2);
  if (!kEnds && a.split && mine) load_states(a.ends, chain_row, at.n0, d.N, h);
  const float* from = a.split && !kEnds ? a.old_state : d.state;
  float sum = 0.f;
  bool fresh = false;                                              // a sequence began inside

  // the piece of 8 channels of a row that this thread stages and finishes
  const int piece_row = threadIdx.x / (Ti::kCh / 8), piece = (threadIdx.x % (Ti::kCh / 8)) * 8;
  const int pch = blockIdx.x * Ti::kCh + piece;
  const bool has_piece = threadIdx.x < Ti::kPieces && pch < d.D;
  const bool wide = a.wide;
  const Rows<T> x = view<T>(d.x), dt = view<T>(d.dt), z = view<T>(d.z), out = view<T>(d.out);
  float bias[8], skip[8];
#pragma unroll
  for (int v = 0; v < 8; ++v) {
    const bool in = has_piece && pch + v < d.D;
    bias[v] = in && d.dt_bias.data ? static_cast<const float*>(d.dt_bias.data)[p * d.dt_bias.stride + pch + v] : 0.f;
    skip[v] = in && d.skip.data ? static_cast<const float*>(d.skip.data)[p * d.skip.stride + pch + v] : 0.f;
  }
  Pack<T, 8> rx, rdt, rz;
  bool live = false;
  auto fetch = [&](int base) {
    const int t = base + piece_row;
    live = has_piece && row_lives(a, p, r, t);
    if (!live) return;
    load8<T>(rx, x.row(p, t), pch, d.D, wide);
    load8<T>(rdt, dt.row(p, t), pch, d.D, wide);
    if (!kEnds && d.z.data) load8<T>(rz, z.row(p, t), pch, d.D, wide);
  };
  if (r.base < r.t1) fetch(r.base);
  const int64_t groups = (a.q.T + kGroup - 1) / kGroup;
  for (int base = r.base; base < r.t1; base += Ti::kRows) {
    // stage
    if (threadIdx.x < Ti::kPieces) {
      float fx[8] = {}, fd[8] = {};
      if (live) {
        rx.get(fx);
        rdt.get(fd);
      }
      float2* dst = s_dd + piece_row * Ti::kCh + piece;
#pragma unroll
      for (int v = 0; v < 8; v += 2) {
        float e;
        const float d0 = live ? softplus(fd[v] + bias[v], e) : 0.f, d1 = live ? softplus(fd[v + 1] + bias[v + 1], e) : 0.f;
        *reinterpret_cast<float4*>(dst + v) = make_float4(d0, d0 * fx[v], d1, d1 * fx[v + 1]);
      }
    }
    stage_bc<T, L>(a, p, r, base, d.b, s_b);
    if (!kEnds) stage_bc<T, L>(a, p, r, base, d.c, s_c);
    const bool special = __syncthreads_or(mark_rows<L>(a, p, r, base, s_begin, s_end));
    const Pack<T, 8> kx = rx, kz = rz;
    const bool klive = live;
    if (base + Ti::kRows < r.t1) fetch(base + Ti::kRows);
    // the recurrence
#pragma unroll 2
    for (int t4 = 0; t4 < Ti::kRows; t4 += 4) {
      if (!kEnds && d.saved && t4 % kGroup == 0 && mine && base + t4 >= r.t0 && base + t4 < r.t1)
        store_states(d.saved, ((int64_t)p * groups + (base + t4) / kGroup) * d.D + at.ch, at.n0, d.N, h);
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = t4 + i;
        if (special) {
          const int s = s_begin[t];
          if (s >= 0) {
            fresh = true;
#pragma unroll
            for (int k = 0; k < kQuad; ++k) h[k] = 0.f;
            if (d.state && mine) {
              const int64_t row = ((int64_t)p * a.q.S + s) * d.D + at.ch;
              load_states(from, row, at.n0, d.N, h);
              if (kEnds) store_states(a.old_state, row, at.n0, d.N, h);
            }
          }
        }
        const float2 dd = s_dd[t * Ti::kCh + at.local];
        const float4 B = *reinterpret_cast<const float4*>(s_b + t * Ti::kN + at.n0);
        h[0] = fmaf(ex2(dd.x * A2[0]), h[0], dd.y * B.x);
        h[1] = fmaf(ex2(dd.x * A2[1]), h[1], dd.y * B.y);
        h[2] = fmaf(ex2(dd.x * A2[2]), h[2], dd.y * B.z);
        h[3] = fmaf(ex2(dd.x * A2[3]), h[3], dd.y * B.w);
        if (kEnds) {
          sum += dd.x;
        } else {
          const float4 C = *reinterpret_cast<const float4*>(s_c + t * Ti::kN + at.n0);
          y[i] = fmaf(C.x, h[0], fmaf(C.y, h[1], fmaf(C.z, h[2], C.w * h[3])));
          if (special && d.state && mine && s_end[t] >= 0)
            store_states(d.state, ((int64_t)p * a.q.S + s_end[t]) * d.D + at.ch, at.n0, d.N, h);
        }
      }
      if (!kEnds) {
        sum_states<L>(y, lane);                                    // every lane of the channel has read these rows
        if (L == 2) {
          s_dd[(t4 + 2 * (lane & 1)) * Ti::kCh + at.local].x = y[0];
          s_dd[(t4 + 2 * (lane & 1) + 1) * Ti::kCh + at.local].x = y[1];
        } else if (lane % L < 4) {
          s_dd[(t4 + row_of(lane)) * Ti::kCh + at.local].x = y[0];
        }
      }
    }
    __syncthreads();
    if (kEnds) continue;
    // finish: the thread reads and later overwrites its own piece of s_dd only
    if (klive) {
      float fx[8], fz[8], o[8];
      kx.get(fx);
      if (d.z.data) kz.get(fz);
      const float2* src = s_dd + piece_row * Ti::kCh + piece;
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        o[v] = fmaf(skip[v], fx[v], src[v].x);
        if (d.z.data) o[v] *= fz[v] * sigmoid(fz[v]);
      }
      store8<T>(o, out.row(p, base + piece_row), pch, d.D, wide);
    }
  }
  if (kEnds && mine) {
    store_states(a.ends, chain_row, at.n0, d.N, h);
    if (at.n0 == 0) a.sums[chain_row] = fresh ? -1.f : sum;
  }
}

// Sequences of one row each: a thread takes 4 states of a channel of one sequence, read and written once.
template <typename T, int L>
__global__ void __launch_bounds__(kThreads) single_kernel(const __grid_constant__ Args a) {
  pdl_wait();
  pdl_launch_dependents();
  const int p = blockIdx.z, lane = threadIdx.x & 31;
  const lsgd_scan_desc& d = a.d;
  const Place<L> at(blockIdx.x, d.D);
  const bool mine = has_states<L>(at, d.N);
  float A2[kQuad];
  decay_rates<L>(a, p, at, A2);
  const float bias = at.in && d.dt_bias.data ? static_cast<const float*>(d.dt_bias.data)[p * d.dt_bias.stride + at.ch] : 0.f;
  const float skip = at.in && d.skip.data ? static_cast<const float*>(d.skip.data)[p * d.skip.stride + at.ch] : 0.f;
  auto one = [&](const lsgd_rows& m, int t, int i, bool in) {
    float f = 0.f;
    if (in) {
      Pack<T, 1> k;
      k.load(view<T>(m).row(p, t) + i);
      k.get(&f);
    }
    return f;
  };
  for (int t = blockIdx.y; t < a.q.S; t += gridDim.y) {
    const int64_t row = ((int64_t)p * a.q.S + t) * d.D + at.ch;
    float h[kQuad] = {};
    if (d.state && mine) load_states(d.state, row, at.n0, d.N, h);
    const float x = one(d.x, t, at.ch, at.in), z = one(d.z, t, at.ch, at.in && d.z.data);
    float e;
    const float delta = softplus(one(d.dt, t, at.ch, at.in) + bias, e), du = delta * x;
    float y = 0.f;
#pragma unroll
    for (int k = 0; k < kQuad; ++k) {
      const bool in = at.n0 + k < d.N;
      h[k] = fmaf(ex2(delta * A2[k]), h[k], du * one(d.b, t, at.n0 + k, in));
      y = fmaf(one(d.c, t, at.n0 + k, in), h[k], y);
    }
    if (d.state && mine) store_states(d.state, row, at.n0, d.N, h);
#pragma unroll
    for (int m = 1; m < L; m *= 2) y += __shfl_xor_sync(0xFFFFFFFFu, y, m);
    if (lane % L == 0 && at.in) {
      float o = fmaf(skip, x, y);
      if (d.z.data) o *= z * sigmoid(z);
      Pack<T, 1> k;
      k.set(&o);
      k.store(view<T>(d.out).row(p, t) + at.ch);
    }
  }
}

// ------------------------------------------------------------------------------------------------ backward
// kEnds: only what the chain's rows add to the adjoint in front of it, and its summed time steps.
template <typename T, int L>
struct BackSmem {
  static constexpr int kRow = Tile<L>::kRows * Tile<L>::kCh, kBc = Tile<L>::kRows * Tile<L>::kN;
  static constexpr int kPart = 8 * kGroup * 8 * L;                 // warps x rows x (4 dB, 4 dC) x L
  static constexpr size_t bytes = sizeof(float) * (3 * kRow + 2 * kBc + 2 * kPart) + 2 * sizeof(int) * Tile<L>::kRows;
};

// Sums of 8 values over the 32 / L channels of a warp; a lane ends up with `count` of them, from `first` on.
template <int L>
struct ChannelSum {
  static constexpr int kCount = L == 16 ? 4 : L == 8 ? 2 : 1;
  static __device__ __forceinline__ int first(int lane) {
    int i = (lane & L) ? 4 : 0;
    if (2 * L <= 16) i += (lane & (2 * L)) ? 2 : 0;
    if (4 * L <= 16) i += (lane & (4 * L)) ? 1 : 0;
    return i;
  }
  static __device__ __forceinline__ void run(float (&v)[8], int lane) {
    halve<4>(v, lane, L);
    if (2 * L <= 16) halve<2>(v, lane, 2 * L);
    if (4 * L <= 16) halve<1>(v, lane, 4 * L);
    if (8 * L <= 16) v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], 8 * L);
  }
  template <int H>
  static __device__ __forceinline__ void halve(float (&v)[8], int lane, int m) {
    const bool up = lane & m;
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const float send = up ? v[i] : v[i + H], keep = up ? v[i + H] : v[i];
      v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, m);
    }
  }
};

template <typename T, int L, bool kEnds>
__global__ void __launch_bounds__(kThreads, kEnds ? 3 : 2) backward_kernel(const __grid_constant__ Args a) {
  using Ti = Tile<L>;
  using Sm = BackSmem<T, L>;
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ __align__(16) float smem[];
  float* s_delta = smem;                                           // then sum q A
  float* s_x = s_delta + Sm::kRow;                                 // then sum g B
  float* s_d = s_x + Sm::kRow;                                     // then sum C h
  float* s_b = s_d + Sm::kRow;
  float* s_c = s_b + Sm::kBc;
  float* s_part = s_c + Sm::kBc;
  int* s_begin = reinterpret_cast<int*>(s_part + 2 * Sm::kPart);
  int* s_end = s_begin + Ti::kRows;
  const int p = blockIdx.z, c = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Range r(a, p, c);
  const lsgd_scan_desc& d = a.d;
  const Place<L> at(blockIdx.x, d.D);
  const bool mine = has_states<L>(at, d.N);
  const int64_t chain_row = ((int64_t)p * a.chains + c) * d.D + at.ch;
  float A2[kQuad], carry[kQuad] = {}, dA[kQuad] = {};              // carry: a_(t+1) g_(t+1)
  decay_rates<L>(a, p, at, A2);
  if (!kEnds && a.split && mine) load_states(a.ends, chain_row, at.n0, d.N, carry);
  float sum = 0.f;
  bool fresh = false;

  const int piece_row = threadIdx.x / (Ti::kCh / 8), piece = (threadIdx.x % (Ti::kCh / 8)) * 8;
  const int pch = blockIdx.x * Ti::kCh + piece;
  const bool has_piece = threadIdx.x < Ti::kPieces && pch < d.D;
  const bool wide = a.wide;
  const Rows<T> x = view<T>(d.x), dt = view<T>(d.dt), z = view<T>(d.z), up = view<T>(d.d_out);
  float bias[8], skip[8], d_skip[8] = {}, d_bias[8] = {};
#pragma unroll
  for (int v = 0; v < 8; ++v) {
    const bool in = has_piece && pch + v < d.D;
    bias[v] = in && d.dt_bias.data ? static_cast<const float*>(d.dt_bias.data)[p * d.dt_bias.stride + pch + v] : 0.f;
    skip[v] = in && d.skip.data ? static_cast<const float*>(d.skip.data)[p * d.skip.stride + pch + v] : 0.f;
  }
  const int64_t groups = (a.q.T + kGroup - 1) / kGroup;
  const int n_tiles = r.base < r.t1 ? (r.t1 - r.base + Ti::kRows - 1) / Ti::kRows : 0;
  int buf = 0;
  for (int it = n_tiles - 1; it >= 0; --it) {
    const int base = r.base + it * Ti::kRows, prow = base + piece_row;
    const bool live = has_piece && row_lives(a, p, r, prow);
    if (threadIdx.x < Ti::kPieces) {
      float fx[8] = {}, fd[8] = {}, fu[8] = {}, fz[8];
      if (live) {
        Pack<T, 8> k;
        if (!kEnds) {
          load8<T>(k, x.row(p, prow), pch, d.D, wide);
          k.get(fx);
        }
        load8<T>(k, dt.row(p, prow), pch, d.D, wide);
        k.get(fd);
        load8<T>(k, up.row(p, prow), pch, d.D, wide);
        k.get(fu);
        if (d.z.data) {
          load8<T>(k, z.row(p, prow), pch, d.D, wide);
          k.get(fz);
        }
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          float e;
          fd[v] = softplus(fd[v] + bias[v], e);
          if (d.z.data) fu[v] *= fz[v] * sigmoid(fz[v]);
        }
      }
      const int o = piece_row * Ti::kCh + piece;
#pragma unroll
      for (int v = 0; v < 8; v += 4) {
        *reinterpret_cast<float4*>(s_delta + o + v) = make_float4(fd[v], fd[v + 1], fd[v + 2], fd[v + 3]);
        if (!kEnds) *reinterpret_cast<float4*>(s_x + o + v) = make_float4(fx[v], fx[v + 1], fx[v + 2], fx[v + 3]);
        *reinterpret_cast<float4*>(s_d + o + v) = make_float4(fu[v], fu[v + 1], fu[v + 2], fu[v + 3]);
      }
    }
    if (!kEnds) stage_bc<T, L>(a, p, r, base, d.b, s_b);
    stage_bc<T, L>(a, p, r, base, d.c, s_c);
    const bool special = __syncthreads_or(mark_rows<L>(a, p, r, base, s_begin, s_end));
    if (kEnds) {
#pragma unroll 4
      for (int t = Ti::kRows - 1; t >= 0; --t) {
        const float delta = s_delta[t * Ti::kCh + at.local], g0 = s_d[t * Ti::kCh + at.local];
        const float4 C = *reinterpret_cast<const float4*>(s_c + t * Ti::kN + at.n0);
        carry[0] = ex2(delta * A2[0]) * fmaf(C.x, g0, carry[0]);
        carry[1] = ex2(delta * A2[1]) * fmaf(C.y, g0, carry[1]);
        carry[2] = ex2(delta * A2[2]) * fmaf(C.z, g0, carry[2]);
        carry[3] = ex2(delta * A2[3]) * fmaf(C.w, g0, carry[3]);
        sum += delta;
        if (special && s_begin[t] >= 0) {
          fresh = true;
#pragma unroll
          for (int k = 0; k < kQuad; ++k) carry[k] = 0.f;
        }
      }
      __syncthreads();
      continue;
    }
    for (int g8 = Ti::kRows / kGroup - 1; g8 >= 0; --g8) {
      const int row0 = base + g8 * kGroup;
      if (row0 >= r.t1 || row0 + kGroup <= r.t0) continue;         // the same for the whole block
      float hs[kGroup][kQuad], as[kGroup][kQuad], first[kQuad] = {}, y[kGroup], gb[kGroup], sa[kGroup];
      if (mine && row0 >= r.t0) load_states(d.saved, ((int64_t)p * groups + row0 / kGroup) * d.D + at.ch, at.n0, d.N, first);
      float h[kQuad];
#pragma unroll
      for (int k = 0; k < kQuad; ++k) h[k] = first[k];
#pragma unroll
      for (int i = 0; i < kGroup; ++i) {
        const int t = g8 * kGroup + i;
        if (special && s_begin[t] >= 0) {
#pragma unroll
          for (int k = 0; k < kQuad; ++k) h[k] = 0.f;
        }
        const float delta = s_delta[t * Ti::kCh + at.local], du = delta * s_x[t * Ti::kCh + at.local];
        const float4 B4 = *reinterpret_cast<const float4*>(s_b + t * Ti::kN + at.n0);
        const float4 C4 = *reinterpret_cast<const float4*>(s_c + t * Ti::kN + at.n0);
        const float B[4] = {B4.x, B4.y, B4.z, B4.w}, C[4] = {C4.x, C4.y, C4.z, C4.w};
        y[i] = 0.f;
#pragma unroll
        for (int k = 0; k < kQuad; ++k) {
          as[i][k] = ex2(delta * A2[k]);
          h[k] = fmaf(as[i][k], h[k], du * B[k]);
          hs[i][k] = h[k];
          y[i] = fmaf(C[k], h[k], y[i]);
        }
      }
      float* part = s_part + buf * Sm::kPart + warp * kGroup * 8 * L;
#pragma unroll
      for (int i = kGroup - 1; i >= 0; --i) {
        const int t = g8 * kGroup + i;
        const bool begins = special && s_begin[t] >= 0;
        const float delta = s_delta[t * Ti::kCh + at.local], du = delta * s_x[t * Ti::kCh + at.local], dy = s_d[t * Ti::kCh + at.local];
        const float4 B4 = *reinterpret_cast<const float4*>(s_b + t * Ti::kN + at.n0);
        const float4 C4 = *reinterpret_cast<const float4*>(s_c + t * Ti::kN + at.n0);
        const float B[4] = {B4.x, B4.y, B4.z, B4.w}, C[4] = {C4.x, C4.y, C4.z, C4.w};
        float v[8];
        gb[i] = sa[i] = 0.f;
#pragma unroll
        for (int k = 0; k < kQuad; ++k) {
          const float g = fmaf(C[k], dy, carry[k]);
          v[k] = g * du;
          v[4 + k] = dy * hs[i][k];
          gb[i] = fmaf(g, B[k], gb[i]);
          carry[k] = begins ? 0.f : as[i][k] * g;
          const float q = begins ? 0.f : carry[k] * (i > 0 ? hs[i > 0 ? i - 1 : 0][k] : first[k]);
          dA[k] = fmaf(q, delta, dA[k]);
          sa[i] = fmaf(q, A2[k], sa[i]);
        }
        ChannelSum<L>::run(v, lane);
        const int f = ChannelSum<L>::first(lane);
        if (8 * L > 16 || !(lane & (8 * L))) {
#pragma unroll
          for (int j = 0; j < ChannelSum<L>::kCount; ++j) part[(i * 8 + f + j) * L + lane % L] = v[j];
        }
      }
      // the sums over the states, where the rows that every lane of the channel has read were
#pragma unroll
      for (int half = 0; half < kGroup; half += 4) {
        float s0[4], s1[4], s2[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) s0[i] = sa[half + i], s1[i] = gb[half + i], s2[i] = y[half + i];
        sum_states<L>(s0, lane);
        sum_states<L>(s1, lane);
        sum_states<L>(s2, lane);
        const int t = g8 * kGroup + half;
        if (L == 2) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int o = (t + 2 * (lane & 1) + i) * Ti::kCh + at.local;
            s_delta[o] = s0[i], s_x[o] = s1[i], s_d[o] = s2[i];
          }
        } else if (lane % L < 4) {
          const int o = (t + row_of(lane)) * Ti::kCh + at.local;
          s_delta[o] = s0[0], s_x[o] = s1[0], s_d[o] = s2[0];
        }
      }
      __syncthreads();
      // the block's sums over its channels, the warps' in order
      for (int i = threadIdx.x; i < kGroup * 8 * L; i += kThreads) {
        const int row = row0 + i / (8 * L), which = (i / L) % 8, n = (i % L) * kQuad + which % 4;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) s += s_part[buf * Sm::kPart + w * kGroup * 8 * L + i];
        if (n < d.N && row >= r.t0 && row < r.t1)
          a.part_bc[((((int64_t)p * a.tiles + blockIdx.x) * a.q.T + row) * 2 + which / 4) * d.N + n] = s;
      }
      buf ^= 1;
    }
    __syncthreads();
    if (live) {
      Pack<T, 8> k;
      float fx[8], fd[8], fu[8], fz[8], o_x[8], o_dt[8], o_z[8];
      load8<T>(k, x.row(p, prow), pch, d.D, wide);
      k.get(fx);
      load8<T>(k, dt.row(p, prow), pch, d.D, wide);
      k.get(fd);
      load8<T>(k, up.row(p, prow), pch, d.D, wide);
      k.get(fu);
      if (d.z.data) {
        load8<T>(k, z.row(p, prow), pch, d.D, wide);
        k.get(fz);
      }
      const int o = piece_row * Ti::kCh + piece;
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        float e;
        const float pre = fd[v] + bias[v], delta = softplus(pre, e);
        const float gB = s_x[o + v], qA = s_delta[o + v] * kLn2, y = fmaf(skip[v], fx[v], s_d[o + v]);
        float g = fu[v];
        if (d.z.data) {
          const float sg = sigmoid(fz[v]), sl = fz[v] * sg;
          o_z[v] = g * y * fmaf(sl, 1.f - sg, sg);
          g *= sl;
        }
        o_x[v] = fmaf(delta, gB, skip[v] * g);
        o_dt[v] = fmaf(fx[v], gB, qA) * __fdividef(pre >= 0.f ? 1.f : e, 1.f + e);
        d_skip[v] = fmaf(g, fx[v], d_skip[v]);
        d_bias[v] += o_dt[v];
      }
      store8<T>(o_x, view<T>(d.dx).row(p, prow), pch, d.D, wide);
      store8<T>(o_dt, view<T>(d.d_dt).row(p, prow), pch, d.D, wide);
      if (d.z.data) store8<T>(o_z, view<T>(d.dz).row(p, prow), pch, d.D, wide);
    }
    __syncthreads();
  }
  if (kEnds) {
    if (mine) {
      store_states(a.ends, chain_row, at.n0, d.N, carry);
      if (at.n0 == 0) a.sums[chain_row] = fresh ? -1.f : sum;
    }
    return;
  }
  if (mine) {
#pragma unroll
    for (int k = 0; k < kQuad; ++k) dA[k] *= A2[k] * kLn2;
    store_states(a.part_a, chain_row, at.n0, d.N, dA);
  }
  // the rows' sums of d skip and d dt_bias, in order
  if (threadIdx.x < Ti::kPieces) {
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      s_x[piece_row * Ti::kCh + piece + v] = d_skip[v];
      s_d[piece_row * Ti::kCh + piece + v] = d_bias[v];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * Ti::kCh; i += kThreads) {
    const int which = i / Ti::kCh, ch = i % Ti::kCh;
    const float* src = which ? s_d : s_x;
    float s = 0.f;
#pragma unroll 8
    for (int row = 0; row < Ti::kRows; ++row) s += src[row * Ti::kCh + ch];
    const int col = blockIdx.x * Ti::kCh + ch;
    if (col < d.D) a.part_v[(((int64_t)p * a.chains + c) * 2 + which) * d.D + col] = s;
  }
}

// db and dc: the channel blocks' sums in order.
template <typename T>
__global__ void __launch_bounds__(256) join_bc_kernel(const __grid_constant__ Args a) {
  pdl_wait();
  pdl_launch_dependents();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n2 = 2 * a.d.N;
  const int p = blockIdx.y;
  if (i >= (int64_t)a.q.T * n2) return;
  const int t = (int)(i / n2), which = (int)(i % n2) / a.d.N, n = (int)(i % n2) % a.d.N;
  if (a.q.starts && a.q.code(p, t) < 0) return;
  const float* src = a.part_bc + (int64_t)p * a.tiles * a.q.T * n2 + i;
  float s = 0.f;
#pragma unroll 8
  for (uint32_t k = 0; k < a.tiles; ++k) s += src[(int64_t)k * a.q.T * n2];
  Pack<T, 1> one;
  one.set(&s);
  one.store(view<T>(which ? a.d.dc : a.d.db).row(p, t) + n);
}

struct Launch {
  int L;
  bool single;
  dim3 grid;
};
cudaError_t launch_forward_f32(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_forward_bf16(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_backward_f32(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_backward_bf16(const Args& a, const Launch& l, cudaStream_t s);
// split: from what every chain adds to what every chain starts from, forwards or backwards (scan.cu)
cudaError_t launch_chain_join(const Args& a, bool reverse, cudaStream_t s);

template <typename T, int L>
cudaError_t forward_of(const Args& a, const Launch& l, cudaStream_t s) {
  if (l.single) return launch_pdl(single_kernel<T, L>, l.grid, dim3(kThreads), 0, s, a);
  if (a.split) {
    cudaError_t e = launch_pdl(forward_kernel<T, L, true>, l.grid, dim3(kThreads), 0, s, a);
    if (e == cudaSuccess) e = launch_chain_join(a, false, s);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(forward_kernel<T, L, false>, l.grid, dim3(kThreads), 0, s, a);
}
template <typename T, int L>
cudaError_t backward_of(const Args& a, const Launch& l, cudaStream_t s) {
  constexpr size_t smem = BackSmem<T, L>::bytes;
  static OncePerDevice attr;
  if (!attr.here()) {
    cudaError_t e = cudaFuncSetAttribute(backward_kernel<T, L, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(backward_kernel<T, L, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    attr.here() = true;
  }
  cudaError_t e = cudaSuccess;
  if (a.split) {
    e = launch_pdl(backward_kernel<T, L, true>, l.grid, dim3(kThreads), smem, s, a);
    if (e == cudaSuccess) e = launch_chain_join(a, true, s);
  }
  if (e == cudaSuccess) e = launch_pdl(backward_kernel<T, L, false>, l.grid, dim3(kThreads), smem, s, a);
  if (e != cudaSuccess) return e;
  const int64_t values = (int64_t)a.q.T * 2 * a.d.N;
  return launch_pdl(join_bc_kernel<T>, dim3((unsigned)((values + 255) / 256), a.d.P), dim3(256), 0, s, a);
}
template <typename T>
cudaError_t forward_any(const Args& a, const Launch& l, cudaStream_t s) {
  switch (l.L) {
    case 2: return forward_of<T, 2>(a, l, s);
    case 4: return forward_of<T, 4>(a, l, s);
    case 8: return forward_of<T, 8>(a, l, s);
    default: return forward_of<T, 16>(a, l, s);
  }
}
template <typename T>
cudaError_t backward_any(const Args& a, const Launch& l, cudaStream_t s) {
  switch (l.L) {
    case 2: return backward_of<T, 2>(a, l, s);
    case 4: return backward_of<T, 4>(a, l, s);
    case 8: return backward_of<T, 8>(a, l, s);
    default: return backward_of<T, 16>(a, l, s);
  }
}

}  // namespace scan
}  // namespace lsgd
