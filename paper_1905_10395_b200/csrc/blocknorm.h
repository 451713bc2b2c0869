// The norms at the boundary of two blocks, with the gate and the scaled residual add between them, in one pass:
//
//     u = post_norm ? y r_y w_post : y,   r_y = 1 / sqrt(mean y^2 + eps)
//     x' = alpha x + beta a(gate) u
//     h = x' r_x w_pre,                   r_x = 1 / sqrt(mean x'^2 + eps)
//
// Backward, with n_x = x' r_x, n_y = y r_y (y without a post norm) and up = d_h w_pre:
//
//     g = d_out + r_x (up - n_x mean(up n_x)),    dx = alpha g
//     d_gate = beta g u a',   s = beta g a w_post,   dy = r_y (s - n_y mean(s n_y))    (no post norm: dy = beta g a)
//     d_w_pre = sum over rows of d_h n_x,         d_w_post = sum over rows of beta g a n_y
//
// A channel gate is a constant of its column, as the gains are: beta, a and w_post are one factor c, and the gradients of
// w_post and of a channel gate are both that column's sum of g n_y times constants, so one running sum serves both.
//
// Memory-bound: every tensor is read or written once, a row stays on the SM from its load to its store.  A thread holds 16
// values of a row -- two pieces of 8, 'threads per row' pieces apart -- and keeps the same columns for every row, so factors
// and sums over the rows are its own: factors in its own words of shared memory, sums in registers.  Blocks are persistent
// (one worker each); short rows share a block, the shortest a warp.  Rows are fetched one
// ahead into shared memory, 16 bytes at a time and asynchronously, by the thread that reads them (its warp for fp32 rows), so
// only the sums over a row (a butterfly in the warp, one exchange between the row's warps) make warps wait for each other.
// Arithmetic is on pairs (fma.rn.f32x2), the modes are template
// parameters and addresses are running pointers: issue slots, not memory, bound the first versions of the backward pass.
//
// Rows of any length: where rows do not start on 16-byte boundaries but all tensors share their layout, a block takes every
// 8th row (or a multiple), whose starts all have the same offset phi from a boundary; pieces begin phi columns before the
// row, so all of them are aligned.  Columns behind a row are filled with zeros by the copy, those before it are masked.
#pragma once
#include <cstring>

#include "lm_ops.h"

namespace lsgd {
namespace blocknorm {

using bf16 = __nv_bfloat16;
constexpr int E = 16;        // values of a row that a thread holds, in two halves of 8
// Threads of an SM, which set the registers of one: 80 and 128.  Rows that fill their threads: forward 8 x 2048 x 2048 takes 80
// us, 98 with 896 threads and as long with 640; fewer registers backward spill the sums.  The ragged kernels' extra addresses
// and masks do not all fit: with a gate for each value they spill up to 344 bytes a thread forward and 180 backward (fp32
// activations; 176 and 220 with bf16 ones beside an fp32 residual, at most 20 with a bf16 residual).
constexpr int kForwardThreads = 768, kBackwardThreads = 512;

struct Args {
  lsgd_blocknorm_desc d;
  uint32_t T;
  int tpr;                   // threads of a row
  int rpb;                   // rows of a block at a time
  int slots;                 // rows in shared memory: 2, or (where two do not fit, and for kDirect) 1
  int phased;                // rows start off 16-byte boundaries
  float inv_d;
  uint32_t blocks_w;         // blocks of one worker
  float* part;               // backward: [P][blocks_w][2][D]
};

// What a launch computes.  kRagged: some thread's 16 columns are not all in the row.  kDirect: any strides, values moved one
// at a time, the mode read from the arguments.
enum : int { kPre = 1, kY = 2, kPost = 4, kToken = 8, kRagged = 16, kDirect = -1 };
inline __host__ __device__ int mode_of(const lsgd_blocknorm_desc& d) {
  return (d.w_pre.data ? kPre : 0) | (d.y.data ? kY : 0) | (d.post_norm ? kPost : 0) | (d.gate_kind == LSGD_GATE_TOKEN ? kToken : 0);
}

// one file per pair of types (residual, activations); mode kDirect or mode_of()
struct Launch {
  int threads, mode;
  size_t smem;
  bool backward;
};
cudaError_t launch_f32_f32(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_f32_bf16(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_bf16_bf16(const Args& a, const Launch& l, cudaStream_t s);
constexpr int kSmemMax = 224 * 1024;      // dynamic shared memory of a block at most

#if defined(__CUDACC__)
// ---- the gate, for the kernels of the rows and of the last sums alike
// 1 / (1 + 2^(-z log2 e)) with the approximate power and reciprocal, each within about 2^-22; the product's rounding adds |z| 2^-24
// to the power.  Subnormal intermediates are flushed: they only move results by less than 2^-126.
__device__ __forceinline__ float sigmoid(float z) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}
__device__ __forceinline__ float gate_slope(float a, int act) {
  if (act == LSGD_GATE_SIGMOID) return a * (1.f - a);
  if (act == LSGD_GATE_TANH) return 1.f - a * a;
  return 1.f;
}
__device__ __forceinline__ float gate_value(float z, int act) {
  return act == LSGD_GATE_SIGMOID ? sigmoid(z) : act == LSGD_GATE_TANH ? tanhf(z) : z;
}
#endif

#if defined(LSGD_BLOCKNORM_KERNELS)
namespace {

#define LSGD_EACH(k) _Pragma("unroll") for (int k = 0; k < 4; ++k)

// ---- a thread's columns: half h covers col[h] .. col[h] + 7; columns outside [0, D) are foreign
struct Cols {
  int col[2], D, gap;
  int have[2];               // columns of the half before the row's end: 0 .. 8
  bool full[2];
  int g, L;                  // this thread among the L of its warp that hold the same row
  __device__ __forceinline__ Cols(int t, int tpr, int D_, int phi) : D(D_), gap(tpr * 8) {
    L = tpr < 32 ? tpr : 32;
    g = (threadIdx.x & 31) % L;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      col[h] = (h * tpr + t) * 8 - phi;
      have[h] = max(0, min(8, D - col[h]));
      full[h] = col[h] >= 0 && have[h] == 8;
    }
  }
  __device__ __forceinline__ bool in(int h, int k) const { return (unsigned)(col[h] + k) < (unsigned)D; }
};

// ---- shared memory of a warp: 16-byte unit u of lane l at [u][l], so units are immediate offsets and a quarter warp is on
// all banks
__device__ __forceinline__ uint4* unit_at(unsigned char* warp, int u) {
  return reinterpret_cast<uint4*>(warp + u * 512 + (threadIdx.x & 31) * 16);
}
// fp32 rows: a half is two units of a thread, 32 bytes in memory.  So that a copy instruction covers whole sectors, the warp
// copies its 64 units (of L lanes: 2 L) in the order of memory, and position n of them holds unit n ^ (n / 8 & 1): a lane's
// two are then read without bank conflicts.
__device__ __forceinline__ uint4* pair_at(unsigned char* warp, int u, int n) {
  return reinterpret_cast<uint4*>(warp + u * 512 + (n ^ (n >> 3 & 1)) * 16);
}
__device__ __forceinline__ void copy16(void* smem, const void* g) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(g) : "memory");
}
// of which the first `bytes` are read and the others become zeros
__device__ __forceinline__ void copy16(void* smem, const void* g, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(g), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <typename T>
constexpr int units() { return (int)sizeof(T) / 2; }   // 16-byte units of a half

template <typename T>
__device__ __forceinline__ T* row_of(const lsgd_rows& r, uint32_t w, uint32_t t) {
  return static_cast<T*>(r.data) + w * r.stride + t * r.ld;
}
// Half h of a row, `p` at the thread's first column of it.
template <typename T, bool RAGGED>
__device__ __forceinline__ void fetch_half(unsigned char* warp, int u, const T* p, const Cols& c, int h) {
  if constexpr (sizeof(T) == 2) {
    if (!RAGGED) copy16(unit_at(warp, u), p);
    else copy16(unit_at(warp, u), p, c.have[h] * 2);
  } else {
    const T* q = p - c.g * 4;             // the g-th unit of the row's part in this warp
    const int n = 2 * (int)(threadIdx.x & 31) - c.g;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (!RAGGED) {
        copy16(pair_at(warp, u, n + i * c.L), q + i * c.L * 4);
      } else {
        const int k = max(0, min(4, c.D - (c.col[h] + (i * c.L - c.g) * 4)));
        copy16(pair_at(warp, u, n + i * c.L), k ? q + i * c.L * 4 : p, k * 4);
      }
    }
  }
}
template <typename T>
__device__ __forceinline__ void zero_half(unsigned char* warp, int u) {
#pragma unroll
  for (int i = 0; i < units<T>(); ++i)
    *(sizeof(T) == 2 ? unit_at(warp, u) : pair_at(warp, u, 2 * (threadIdx.x & 31) + i)) = make_uint4(0, 0, 0, 0);
}
template <typename T, bool RAGGED>
__device__ __forceinline__ void take_half(unsigned char* warp, int u, const Cols& c, int h, float2 (&f)[4]) {
  uint4 v[units<T>()];
#pragma unroll
  for (int i = 0; i < units<T>(); ++i) v[i] = *(sizeof(T) == 2 ? unit_at(warp, u) : pair_at(warp, u, 2 * (threadIdx.x & 31) + i));
  float* e = reinterpret_cast<float*>(f);
  if constexpr (sizeof(T) == 2) {
    Pack<T, 8> p;
    p.a = v[0];
    p.get(e);
  } else {
    memcpy(e, v, sizeof(v));
  }
  if (RAGGED && c.col[h] < 0) {
    LSGD_EACH(k) {
      if (c.col[h] + 2 * k < 0) f[k].x = 0.f;
      if (c.col[h] + 2 * k + 1 < 0) f[k].y = 0.f;
    }
  }
}
template <typename T, bool DIRECT, bool RAGGED>
__device__ __forceinline__ void store_half(T* p, const Cols& c, int h, bool live, const float2 (&f)[4]) {
  if (!live) return;
  if (!DIRECT && (!RAGGED || c.full[h])) {
    Pack<T, 8> o;
    o.set(reinterpret_cast<const float*>(f));
    o.store(p);
  } else {
    LSGD_EACH(k) {
      Pack<T, 1> e;
      e.set(&f[k].x);
      if (c.in(h, 2 * k)) e.store(p + 2 * k);
      e.set(&f[k].y);
      if (c.in(h, 2 * k + 1)) e.store(p + 2 * k + 1);
    }
  }
}

// fp32 vectors, aligned to their element only; 0 at foreign columns
__device__ __forceinline__ void vector_half(const float* v, const Cols& c, int h, float2 (&f)[4]) {
  LSGD_EACH(k) {
    f[k].x = c.in(h, 2 * k) ? __ldg(v + c.col[h] + 2 * k) : 0.f;
    f[k].y = c.in(h, 2 * k + 1) ? __ldg(v + c.col[h] + 2 * k + 1) : 0.f;
  }
}
__device__ __forceinline__ void keep_half(unsigned char* warp, int u, const float2 (&f)[4]) {
#pragma unroll
  for (int q = 0; q < 2; ++q)
    *reinterpret_cast<float4*>(unit_at(warp, u + q)) = make_float4(f[2 * q].x, f[2 * q].y, f[2 * q + 1].x, f[2 * q + 1].y);
}
__device__ __forceinline__ void kept_half(unsigned char* warp, int u, float2 (&f)[4]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const float4 v = *reinterpret_cast<const float4*>(unit_at(warp, u + q));
    f[2 * q] = make_float2(v.x, v.y);
    f[2 * q + 1] = make_float2(v.z, v.w);
  }
}

// Sum over the threads of a row; every one of them gets it.  s_red: 16 words per row of the block, zero beyond its warps.
// A row of several warps meets at a named barrier of its own.
__device__ __forceinline__ float row_sum(float2 a, int tpr, int sub, float* s_red) {
  float v = a.x + a.y;
  if (tpr < 32) {
    for (int o = tpr >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  if (tpr == 32) return v;
  float* row = s_red + sub * 16;
  if ((threadIdx.x & 31) == 0) row[((int)threadIdx.x - sub * tpr) >> 5] = v;
  asm volatile("bar.sync %0, %1;" ::"r"(sub + 1), "r"(tpr) : "memory");
  const float4* q = reinterpret_cast<const float4*>(row);
  float s = 0.f;
  for (int i = 0; i < tpr; i += 128) {
    const float4 w = *q++;
    s += (w.x + w.y) + (w.z + w.w);
  }
  return s;
}

__device__ __forceinline__ void gate_values(float2 (&f)[4], int act) {
  if (act == LSGD_GATE_SIGMOID) {
    LSGD_EACH(k) f[k] = make_float2(sigmoid(f[k].x), sigmoid(f[k].y));
  } else if (act == LSGD_GATE_TANH) {
    LSGD_EACH(k) f[k] = make_float2(tanhf(f[k].x), tanhf(f[k].y));
  }
}

__device__ __forceinline__ float* vector_of(const lsgd_rows& r, uint32_t w) { return static_cast<float*>(r.data) + w * r.stride; }
constexpr int kMaxRowsOfBlock = 4;        // rows of more than one warp that share a block
constexpr int kRowWords = kMaxRowsOfBlock * 16;
constexpr int kSums = 4;                  // exchanges in flight: two sums a row, two rows
constexpr int kFactorUnits = 4;           // 16 fp32 values

// c = beta a(channel gate) w_post at a thread's half
__device__ __forceinline__ void factor_half(const Args& a, uint32_t w, const Cols& c, int h, bool post, bool channel, float2 (&f)[4]) {
  LSGD_EACH(k) f[k] = both(a.d.beta);
  float2 v[4];
  if (post) {
    vector_half(vector_of(a.d.w_post, w), c, h, v);
    LSGD_EACH(k) f[k] = mul2(f[k], v[k]);
  }
  if (channel) {
    vector_half(vector_of(a.d.gate, w), c, h, v);
    gate_values(v, a.d.gate_act);
    LSGD_EACH(k) f[k] = mul2(f[k], v[k]);
  }
}

// A tensor that rows are read from: fetched ahead, or read in place.  p: at the first half's first column.
template <typename T, bool DIRECT, bool RAGGED>
struct Input {
  const T* p;
  int64_t step;
  int unit;                               // of the first half in the thread's words
  __device__ __forceinline__ void open(const lsgd_rows& r, uint32_t w, uint32_t t, uint32_t rows, const Cols& c, int unit_) {
    p = row_of<T>(r, w, t) + c.col[0];
    step = (int64_t)rows * r.ld;
    unit = unit_;
  }
  __device__ __forceinline__ void fetch(unsigned char* warp, bool live, const Cols& c) {
    if constexpr (!DIRECT) {
      if (live) {
        fetch_half<T, RAGGED>(warp, unit, p, c, 0);
        fetch_half<T, RAGGED>(warp, unit + units<T>(), p + c.gap, c, 1);
        p += step;
      } else {
        zero_half<T>(warp, unit);
        zero_half<T>(warp, unit + units<T>());
      }
    } else {
      p += step;
    }
  }
  __device__ __forceinline__ void get(unsigned char* warp, bool live, const Cols& c, int h, float2 (&f)[4]) const {
    if constexpr (!DIRECT) {
      take_half<T, RAGGED>(warp, unit + h * units<T>(), c, h, f);
    } else {
      const T* q = p + h * c.gap;
      LSGD_EACH(k) {
        Pack<T, 1> e;
        f[k] = both(0.f);
        if (live && c.in(h, 2 * k)) { e.load(q + 2 * k); e.get(&f[k].x); }
        if (live && c.in(h, 2 * k + 1)) { e.load(q + 2 * k + 1); e.get(&f[k].y); }
      }
    }
  }
};
template <typename T, bool DIRECT, bool RAGGED>
struct Output {
  T* p;
  int64_t step;
  __device__ __forceinline__ void open(const lsgd_rows& r, uint32_t w, uint32_t t, uint32_t rows, const Cols& c) {
    p = row_of<T>(r, w, t) + c.col[0];
    step = (int64_t)rows * r.ld;
  }
  __device__ __forceinline__ void put(const Cols& c, int h, bool live, const float2 (&f)[4]) {
    store_half<T, DIRECT, RAGGED>(p + h * c.gap, c, h, live, f);
  }
  __device__ __forceinline__ void advance() { p += step; }
};

// 8 x 2048 rows of 2048 values, fp32 residual, a sigmoid gate for each value: 80 to 83 us for 470 MB (two devices), 5.9 to 5.7
// TB/s or 0.90 to 0.87 of the measured copy bandwidth.
// Blocks: blockIdx.y = worker; block b of a worker takes its rows b rpb .., then those blocks_w rpb further on.
template <typename TR, typename TA, int MODE>
__global__ void __launch_bounds__(kForwardThreads, 1)
forward_kernel(const __grid_constant__ Args a) {
  constexpr bool DIRECT = MODE == kDirect, RAGGED = DIRECT || (MODE & kRagged);
  constexpr bool PAIRS = !DIRECT && sizeof(TR) == 4;   // lanes read what others of their warp have copied
  pdl_wait();
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ __align__(16) float s_red[kSums * kRowWords];
  const lsgd_blocknorm_desc& d = a.d;
  const int mode = DIRECT ? mode_of(d) : MODE;
  const bool pre = mode & kPre, has_y = mode & kY, post = mode & kPost, token = mode & kToken;
  const bool channel = has_y && d.gate_kind == LSGD_GATE_CHANNEL;
  const int sub = threadIdx.x / a.tpr;
  const uint32_t w = blockIdx.y, step = a.blocks_w * a.rpb;
  uint32_t t = blockIdx.x * a.rpb + sub;
  const int phi = RAGGED && a.phased ? (int)((w * (uint64_t)d.x.stride + t * (uint64_t)d.x.ld) & 7) : 0;
  const Cols c((int)threadIdx.x - sub * a.tpr, a.tpr, d.D, phi);
  // a thread's words: w_pre, c, x, y, gate
  const int u_c = pre ? kFactorUnits : 0, u_x = u_c + (has_y ? kFactorUnits : 0), u_y = u_x + 2 * units<TR>();
  const int u_g = u_y + (has_y ? 2 * units<TA>() : 0), stage = u_g + (token ? 2 * units<TA>() : 0) - u_x;
  const int words = DIRECT ? u_x : u_x + a.slots * stage;
  unsigned char* warp = smem + (threadIdx.x >> 5) * words * 512;
  for (int i = threadIdx.x; i < kSums * kRowWords; i += blockDim.x) s_red[i] = 0.f;
  Input<TR, DIRECT, RAGGED> ix;
  Input<TA, DIRECT, RAGGED> iy, ig;
  Output<TR, DIRECT, RAGGED> ox;
  Output<TA, DIRECT, RAGGED> oh;
  ix.open(d.x, w, t, step, c, u_x);
  if (has_y) iy.open(d.y, w, t, step, c, u_y), ox.open(d.out, w, t, step, c);
  if (token) ig.open(d.gate, w, t, step, c, u_g);
  if (pre) oh.open(d.h, w, t, step, c);
  const auto fetch = [&](uint32_t row, unsigned char* warp) {
    const bool more = row < a.T;
    ix.fetch(warp, more, c);
    if (has_y) iy.fetch(warp, more, c);
    if (token) ig.fetch(warp, more, c);
    copy_commit();
  };
  if (!DIRECT) {
    fetch(t, warp);
  }
  unsigned char* in = warp;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float2 f[4];
    if (pre) {
      vector_half(vector_of(d.w_pre, w), c, h, f);
      keep_half(warp, 2 * h, f);
    }
    if (has_y) {
      factor_half(a, w, c, h, post, channel, f);
      keep_half(warp, u_c + 2 * h, f);
    }
  }
  __syncthreads();
  int phase = 0;
  for (uint32_t t0 = blockIdx.x * a.rpb; t0 < a.T; t0 += step, t += step, phase ^= 2) {
    const bool live = t < a.T;
    unsigned char* next = a.slots == 2 && in == warp ? warp + stage * 512 : warp;
    if (a.slots == 2) {
      fetch(t + step, next);
      copy_wait<1>();
    } else {
      copy_wait<0>();
    }
    if (PAIRS) __syncwarp();
    float2 x[2][4], y[2][4], g[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ix.get(in, live, c, h, x[h]);
      if (has_y) iy.get(in, live, c, h, y[h]);
      if (token) ig.get(in, live, c, h, g[h]);
    }
    if (PAIRS) __syncwarp();              // the words are free again
    if (a.slots == 1) fetch(t + step, in);
    in = next;
    if (has_y) {
      float rs = 1.f;
      if (post) {
        float2 q = both(0.f);
#pragma unroll
        for (int h = 0; h < 2; ++h) LSGD_EACH(k) q = fma2(y[h][k], y[h][k], q);
        rs = rsqrtf(row_sum(q, a.tpr, sub, s_red + phase * kRowWords) * a.inv_d + d.eps);
        if (live && (int)threadIdx.x == sub * a.tpr) d.rstd_post[(size_t)w * a.T + t] = rs;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float2 f[4];
        if (token) {
          gate_values(g[h], d.gate_act);
          LSGD_EACH(k) y[h][k] = mul2(y[h][k], g[h][k]);
        }
        kept_half(warp, u_c + 2 * h, f);
        if (post) {
          LSGD_EACH(k) y[h][k] = mul2(y[h][k], both(rs));
        }
        LSGD_EACH(k) x[h][k] = fma2(f[k], y[h][k], mul2(both(d.alpha), x[h][k]));
        ox.put(c, h, live, x[h]);
      }
      ox.advance();
    }
    if (pre) {
      float2 q = both(0.f);
#pragma unroll
      for (int h = 0; h < 2; ++h) LSGD_EACH(k) q = fma2(x[h][k], x[h][k], q);
      const float rs = rsqrtf(row_sum(q, a.tpr, sub, s_red + (phase + 1) * kRowWords) * a.inv_d + d.eps);
      if (live && (int)threadIdx.x == sub * a.tpr) d.rstd_pre[(size_t)w * a.T + t] = rs;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float2 f[4];
        kept_half(warp, 2 * h, f);
        LSGD_EACH(k) x[h][k] = mul2(mul2(x[h][k], both(rs)), f[k]);
        oh.put(c, h, live, x[h]);
      }
      oh.advance();
    }
  }
  copy_wait<0>();
}

// 16384 rows of 4096 bf16 values, both norms and a channel gate: 139 us for 805 MB, 5.8 TB/s or 0.88 of the copy bandwidth (8
// more for the last sums).  16 warps an SM, bound by registers: the sums of two gains and a row in each thread.
template <typename TR, typename TA, int MODE>
__global__ void __launch_bounds__(kBackwardThreads, 1)
backward_kernel(const __grid_constant__ Args a) {
  constexpr bool DIRECT = MODE == kDirect, RAGGED = DIRECT || (MODE & kRagged);
  constexpr bool PAIRS = !DIRECT && sizeof(TR) == 4;   // lanes read what others of their warp have copied
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ __align__(16) float s_red[kSums * kRowWords];
  const lsgd_blocknorm_desc& d = a.d;
  const int mode = DIRECT ? mode_of(d) : MODE;
  const bool pre = mode & kPre, has_y = mode & kY, post = mode & kPost, token = mode & kToken;
  const bool channel = has_y && d.gate_kind == LSGD_GATE_CHANNEL, has_d = d.d_out.data != nullptr;
  const int sub = threadIdx.x / a.tpr;
  const uint32_t w = blockIdx.y, step = a.blocks_w * a.rpb;
  uint32_t t = blockIdx.x * a.rpb + sub;
  const int phi = RAGGED && a.phased ? (int)((w * (uint64_t)d.dx.stride + t * (uint64_t)d.dx.ld) & 7) : 0;
  const Cols c((int)threadIdx.x - sub * a.tpr, a.tpr, d.D, phi);
  // a thread's words: w_pre, c, d_out, out, d_h, y, gate
  const int u_c = pre ? kFactorUnits : 0, u_d = u_c + (has_y ? kFactorUnits : 0), u_out = u_d + 2 * units<TR>();
  const int u_dh = u_out + (pre ? 2 * units<TR>() : 0), u_y = u_dh + (pre ? 2 * units<TA>() : 0);
  const int u_g = u_y + (has_y ? 2 * units<TA>() : 0), stage = u_g + (token ? 2 * units<TA>() : 0) - u_d;
  const int words = DIRECT ? u_d : u_d + a.slots * stage;
  unsigned char* warp = smem + (threadIdx.x >> 5) * words * 512;
  for (int i = threadIdx.x; i < kSums * kRowWords; i += blockDim.x) s_red[i] = 0.f;
  Input<TR, DIRECT, RAGGED> id, io;
  Input<TA, DIRECT, RAGGED> ih, iy, ig;
  Output<TR, DIRECT, RAGGED> ox;
  Output<TA, DIRECT, RAGGED> oy, og;
  ox.open(d.dx, w, t, step, c);
  if (has_d) id.open(d.d_out, w, t, step, c, u_d);
  if (pre) io.open(d.out, w, t, step, c, u_out), ih.open(d.d_h, w, t, step, c, u_dh);
  if (has_y) iy.open(d.y, w, t, step, c, u_y), oy.open(d.dy, w, t, step, c);
  if (token) ig.open(d.gate, w, t, step, c, u_g), og.open(d.d_gate, w, t, step, c);
  const auto fetch = [&](uint32_t row, unsigned char* warp) {
    const bool more = row < a.T;
    if (has_d) id.fetch(warp, more, c);
    if (pre) {
      io.fetch(warp, more, c);
      ih.fetch(warp, more, c);
    }
    if (has_y) iy.fetch(warp, more, c);
    if (token) ig.fetch(warp, more, c);
    copy_commit();
  };
  if (!DIRECT) fetch(t, warp);
  unsigned char* in = warp;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float2 f[4];
    if (pre) {
      vector_half(vector_of(d.w_pre, w), c, h, f);
      keep_half(warp, 2 * h, f);
    }
    if (has_y) {
      factor_half(a, w, c, h, post, channel, f);
      keep_half(warp, u_c + 2 * h, f);
    }
  }
  __syncthreads();
  float2 sum_pre[2][4], sum_y[2][4];      // of d_h n_x and of g (a) n_y
#pragma unroll
  for (int h = 0; h < 2; ++h) LSGD_EACH(k) sum_pre[h][k] = sum_y[h][k] = both(0.f);
  int phase = 0;
  for (uint32_t t0 = blockIdx.x * a.rpb; t0 < a.T; t0 += step, t += step, phase ^= 2) {
    const bool live = t < a.T;
    const size_t r = (size_t)w * a.T + t;
    // n: normalised rows; up: what arrives at them times the gain -- of the second norm first, then of the first
    float2 n[2][4], up[2][4];
    float rs = 0.f, mean = 0.f, rs_y = 0.f;
    if (pre) rs = live ? d.rstd_pre[r] : 0.f;
    if (post) rs_y = live ? d.rstd_post[r] : 0.f;
    unsigned char* next = a.slots == 2 && in == warp ? warp + stage * 512 : warp;
    if (a.slots == 2) {
      fetch(t + step, next);
      copy_wait<1>();
    } else {
      copy_wait<0>();
    }
    if (PAIRS) __syncwarp();
    if (pre) {
      float2 q = both(0.f);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float2 f[4];
        io.get(in, live, c, h, n[h]);
        ih.get(in, live, c, h, up[h]);
        kept_half(warp, 2 * h, f);
        LSGD_EACH(k) {
          n[h][k] = mul2(n[h][k], both(rs));
          sum_pre[h][k] = fma2(up[h][k], n[h][k], sum_pre[h][k]);
          up[h][k] = mul2(up[h][k], f[k]);
          q = fma2(up[h][k], n[h][k], q);
        }
      }
      mean = -rs * (row_sum(q, a.tpr, sub, s_red + phase * kRowWords) * a.inv_d);
    }
    float2 q = both(0.f);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float2 g[4];                        // d_out, then the gradient of x'
      LSGD_EACH(k) g[k] = both(0.f);
      if (has_d) id.get(in, live, c, h, g);
      if (pre) {
        LSGD_EACH(k) g[k] = fma2(n[h][k], both(mean), fma2(up[h][k], both(rs), g[k]));
      }
      float2 b[4];
      LSGD_EACH(k) b[k] = has_y ? mul2(both(d.alpha), g[k]) : g[k];
      ox.put(c, h, live, b);
      if (!has_y) continue;
      iy.get(in, live, c, h, n[h]);
      if (post) {
        LSGD_EACH(k) n[h][k] = mul2(n[h][k], both(rs_y));
      }
      float2 f[4];
      kept_half(warp, u_c + 2 * h, f);
      if (token) {
        ig.get(in, live, c, h, b);
        gate_values(b, d.gate_act);
        LSGD_EACH(k) {
          const float2 av = b[k];
          b[k] = mul2(mul2(mul2(g[k], n[h][k]), f[k]), make_float2(gate_slope(av.x, d.gate_act), gate_slope(av.y, d.gate_act)));
          g[k] = mul2(g[k], av);
        }
        og.put(c, h, live, b);
      }
      LSGD_EACH(k) {
        sum_y[h][k] = fma2(g[k], n[h][k], sum_y[h][k]);
        up[h][k] = mul2(g[k], f[k]);
        q = fma2(up[h][k], n[h][k], q);
      }
      if (!post) oy.put(c, h, live, up[h]);
    }
    if (PAIRS) __syncwarp();              // the words are free again
    if (a.slots == 1) fetch(t + step, in);
    in = next;
    if (post) {
      mean = -rs_y * (row_sum(q, a.tpr, sub, s_red + (phase + 1) * kRowWords) * a.inv_d);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        LSGD_EACH(k) up[h][k] = fma2(n[h][k], both(mean), mul2(up[h][k], both(rs_y)));
        oy.put(c, h, live, up[h]);
      }
    }
    ox.advance();
    oy.advance();
    og.advance();
  }
  copy_wait<0>();
  // one partial row per block for the two sums
  float* s_sum = reinterpret_cast<float*>(smem);       // [rpb][D]
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const bool want = j == 0 ? pre && d.d_w_pre.data : (post && d.d_w_post.data) || (channel && d.d_gate.data);
    if (!want) continue;
    float* part = a.part + (((size_t)w * a.blocks_w + blockIdx.x) * 2 + j) * d.D;
    float* dst = part;
    if (a.rpb > 1) {
      __syncthreads();                    // the factors and the previous sum have been read
      dst = s_sum + sub * d.D;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) LSGD_EACH(k) {
      const float2 v = j == 0 ? sum_pre[h][k] : sum_y[h][k];
      if (c.in(h, 2 * k)) dst[c.col[h] + 2 * k] = v.x;
      if (c.in(h, 2 * k + 1)) dst[c.col[h] + 2 * k + 1] = v.y;
    }
    if (a.rpb > 1) {                      // add the block's rows in order
      __syncthreads();
      for (int col = threadIdx.x; col < d.D; col += blockDim.x) {
        float v = 0.f;
        for (int q = 0; q < a.rpb; ++q) v += s_sum[q * d.D + col];
        part[col] = v;
      }
    }
  }
}

template <typename TR, typename TA, int MODE>
cudaError_t launch_mode(const Args& a, const Launch& l, cudaStream_t s) {
  static OncePerDevice once;
  if (!once.here()) {
    cudaError_t e = cudaFuncSetAttribute(forward_kernel<TR, TA, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(backward_kernel<TR, TA, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
    if (e != cudaSuccess) return e;
    once.here() = true;
  }
  const dim3 grid(a.blocks_w, a.d.P), block(l.threads);
  return l.backward ? launch_pdl(backward_kernel<TR, TA, MODE>, grid, block, l.smem, s, a)
                    : launch_pdl(forward_kernel<TR, TA, MODE>, grid, block, l.smem, s, a);
}

template <typename TR, typename TA, int RAGGED>
cudaError_t launch_shape(const Args& a, const Launch& l, cudaStream_t s) {
  switch (l.mode & ~kRagged) {
    case kPre: return launch_mode<TR, TA, RAGGED | kPre>(a, l, s);
    case kY: return launch_mode<TR, TA, RAGGED | kY>(a, l, s);
    case kY | kPre: return launch_mode<TR, TA, RAGGED | kY | kPre>(a, l, s);
    case kY | kPost: return launch_mode<TR, TA, RAGGED | kY | kPost>(a, l, s);
    case kY | kPost | kPre: return launch_mode<TR, TA, RAGGED | kY | kPost | kPre>(a, l, s);
    case kY | kToken: return launch_mode<TR, TA, RAGGED | kY | kToken>(a, l, s);
    case kY | kToken | kPre: return launch_mode<TR, TA, RAGGED | kY | kToken | kPre>(a, l, s);
    case kY | kToken | kPost: return launch_mode<TR, TA, RAGGED | kY | kToken | kPost>(a, l, s);
    case kY | kToken | kPost | kPre: return launch_mode<TR, TA, RAGGED | kY | kToken | kPost | kPre>(a, l, s);
    default: return cudaErrorInvalidValue;
  }
}
template <typename TR, typename TA>
cudaError_t launch_types(const Args& a, const Launch& l, cudaStream_t s) {
  if (l.mode == kDirect) return launch_mode<TR, TA, kDirect>(a, l, s);
  return l.mode & kRagged ? launch_shape<TR, TA, kRagged>(a, l, s) : launch_shape<TR, TA, 0>(a, l, s);
}

}  // namespace
#endif  // LSGD_BLOCKNORM_KERNELS

}  // namespace blocknorm
}  // namespace lsgd
