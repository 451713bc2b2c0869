// The norms at the boundary of two blocks, with the gate and the scaled residual add between them, in one pass:
//
//     u = post_norm ? y r_y w_post : y,   r_y = 1 / sqrt(mean y^2 + eps)
//     x' = alpha x + beta a(gate) u
//     h = x' r_x w_pre,                   r_x = 1 / sqrt(mean x'^2 + eps)
//
// Backward, with n_x = x' r_x, n_y = y r_y and up = d_h w_pre:
//
//     d = d_out + r_x (up - n_x mean(up n_x)),    dx = alpha d,    dz = beta d
//     d_gate = dz u a',   s = dz a w_post,        dy = r_y (s - n_y mean(s n_y))    (no post norm: dy = dz a)
//     d_w_pre = sum over rows of d_h n_x,         d_w_post = sum over rows of dz a n_y
//
// Memory-bound: every tensor is read or written once, a row stays in registers from its load to its store.  A thread holds
// 8 values of a row -- a piece of 8 (or pieces of VEC) every 'threads per row' pieces -- and short rows share a block, the
// shortest a warp.  The sums over a row are a butterfly inside the warp, then one shared-memory exchange.
#include "lm_ops.h"

namespace lsgd {
namespace {

using bf16 = __nv_bfloat16;

struct NormArgs {
  lsgd_blocknorm_desc d;
  uint32_t rows_n;           // P T
  uint32_t T;
  int tpr;                   // threads of a row
  int rpb;                   // rows of a block at a time
  float inv_d;
  // backward
  uint32_t blocks_w;         // blocks of one worker
  float* part;               // [P][blocks_w][3][D]
};

template <int VEC, int E>
struct Cols {
  int tpr, t, D;
  __device__ __forceinline__ int col(int i) const { return (i * tpr + t) * VEC; }
  __device__ __forceinline__ bool in(int i) const { return col(i) < D; }
};

template <typename T, int VEC, int E>
__device__ __forceinline__ void load_row(const T* row, const Cols<VEC, E>& c, Pack<T, VEC> (&r)[E / VEC]) {
#pragma unroll
  for (int i = 0; i < E / VEC; ++i)
    if (c.in(i)) r[i].load(row + c.col(i));
}
template <typename T, int VEC, int E>
__device__ __forceinline__ void unpack(const Cols<VEC, E>& c, const Pack<T, VEC> (&r)[E / VEC], float (&f)[E]) {
#pragma unroll
  for (int i = 0; i < E / VEC; ++i) {
    if (c.in(i)) r[i].get(f + i * VEC);
    else {
#pragma unroll
      for (int k = 0; k < VEC; ++k) f[i * VEC + k] = 0.f;
    }
  }
}
template <typename T, int VEC, int E>
__device__ __forceinline__ void read_row(const T* row, const Cols<VEC, E>& c, float (&f)[E]) {
  Pack<T, VEC> r[E / VEC];
  load_row<T, VEC, E>(row, c, r);
  unpack<T, VEC, E>(c, r, f);
}
template <typename T, int VEC, int E>
__device__ __forceinline__ void write_row(T* row, const Cols<VEC, E>& c, const float (&f)[E]) {
#pragma unroll
  for (int i = 0; i < E / VEC; ++i)
    if (c.in(i)) {
      Pack<T, VEC> o;
      o.set(f + i * VEC);
      o.store(row + c.col(i));
    }
}
// fp32 vectors (weights, gates of channels): aligned to their element only
template <int VEC, int E>
__device__ __forceinline__ void read_vector(const float* v, const Cols<VEC, E>& c, float (&f)[E]) {
#pragma unroll
  for (int i = 0; i < E / VEC; ++i)
#pragma unroll
    for (int k = 0; k < VEC; ++k) f[i * VEC + k] = c.in(i) ? __ldg(v + c.col(i) + k) : 0.f;
}

// Sum over the threads of a row; every one of them gets it.  All threads of the block call it.
__device__ __forceinline__ float row_sum(float v, int tpr, float* s_red) {
  const int w = tpr < 32 ? tpr : 32;
  for (int o = w >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  if (tpr <= 32) return v;
  if ((threadIdx.x & 31) == 0) s_red[threadIdx.x >> 5] = v;
  __syncthreads();
  const int w0 = threadIdx.x / tpr * (tpr >> 5), n = tpr >> 5;
  float s = 0.f;
  for (int i = 0; i < n; ++i) s += s_red[w0 + i];
  return s;
}

__device__ __forceinline__ float gate_value(float z, int act) {
  if (act == LSGD_GATE_SIGMOID) return 1.f / (1.f + __expf(-z));
  if (act == LSGD_GATE_TANH) return tanhf(z);
  return z;
}
__device__ __forceinline__ float gate_slope(float a, int act) {
  if (act == LSGD_GATE_SIGMOID) return a * (1.f - a);
  if (act == LSGD_GATE_TANH) return 1.f - a * a;
  return 1.f;
}

__device__ __forceinline__ float* at(const lsgd_rows& r, uint32_t w) { return static_cast<float*>(r.data) + w * r.stride; }
template <typename T>
__device__ __forceinline__ T* at(const lsgd_rows& r, uint32_t w, uint32_t t) {
  return static_cast<T*>(r.data) + w * r.stride + t * r.ld;
}

template <typename TR, typename TA, int VEC>
__global__ void __launch_bounds__(1024)
blocknorm_forward_kernel(const __grid_constant__ NormArgs a) {
  constexpr int E = 8;
  pdl_wait();
  __shared__ float s_red[2][32];
  const lsgd_blocknorm_desc& d = a.d;
  const int sub = threadIdx.x / a.tpr;
  const Cols<VEC, E> c{a.tpr, (int)threadIdx.x - sub * a.tpr, d.D};
  const uint32_t r = blockIdx.x * a.rpb + sub;
  const bool live = r < a.rows_n;
  const uint32_t w = live ? r / a.T : 0, t = live ? r - w * a.T : 0;
  const bool has_y = d.y.data != nullptr, pre = d.w_pre.data != nullptr;
  float x[E];
  if (live) read_row<TR, VEC, E>(at<const TR>(d.x, w, t), c, x);
  else
    for (int k = 0; k < E; ++k) x[k] = 0.f;
  if (has_y) {
    float y[E];
    if (live) read_row<TA, VEC, E>(at<const TA>(d.y, w, t), c, y);
    else
      for (int k = 0; k < E; ++k) y[k] = 0.f;
    float g[E];
    if (live && d.gate_kind == LSGD_GATE_TOKEN) read_row<TA, VEC, E>(at<const TA>(d.gate, w, t), c, g);
    if (live && d.gate_kind == LSGD_GATE_CHANNEL) read_vector<VEC, E>(at(d.gate, w), c, g);
    if (d.post_norm) {
      float q = 0.f;
#pragma unroll
      for (int k = 0; k < E; ++k) q = fmaf(y[k], y[k], q);
      const float rs = rsqrtf(row_sum(q, a.tpr, s_red[0]) * a.inv_d + d.eps);
      if (live) {
        if (c.t == 0) d.rstd_post[r] = rs;
        float wp[E];
        read_vector<VEC, E>(at(d.w_post, w), c, wp);
#pragma unroll
        for (int k = 0; k < E; ++k) y[k] = y[k] * rs * wp[k];
      }
    }
    if (live) {
      if (d.gate_kind != LSGD_GATE_NONE) {
#pragma unroll
        for (int k = 0; k < E; ++k) y[k] *= gate_value(g[k], d.gate_act);
      }
#pragma unroll
      for (int k = 0; k < E; ++k) x[k] = fmaf(d.beta, y[k], d.alpha * x[k]);
#pragma unroll
      for (int i = 0; i < E / VEC; ++i)
        if (!c.in(i))
          for (int k = 0; k < VEC; ++k) x[i * VEC + k] = 0.f;
      write_row<TR, VEC, E>(at<TR>(d.out, w, t), c, x);
    }
  }
  if (pre) {
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < E; ++k) q = fmaf(x[k], x[k], q);
    const float rs = rsqrtf(row_sum(q, a.tpr, s_red[1]) * a.inv_d + d.eps);
    if (live) {
      if (c.t == 0) d.rstd_pre[r] = rs;
      float wp[E];
      read_vector<VEC, E>(at(d.w_pre, w), c, wp);
#pragma unroll
      for (int k = 0; k < E; ++k) x[k] = x[k] * rs * wp[k];
      write_row<TA, VEC, E>(at<TA>(d.h, w, t), c, x);
    }
  }
}

// A thread's own 8 values of a row, fetched ahead into shared memory: the thread that copies them is the one that reads
// them, so no barrier guards the ring, only the thread's own copy groups.  16-byte unit u of a tensor lies at
// [u][thread], which keeps a quarter warp's accesses on all banks.
__device__ __forceinline__ void copy16(void* smem, const void* g) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(g) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <typename T>
constexpr int units() { return sizeof(T) * 8 / 16; }
template <typename T>
__device__ __forceinline__ void fetch_ahead(uint4* ring, int& unit, const T* row, int col) {
#pragma unroll
  for (int u = 0; u < units<T>(); ++u)
    copy16(ring + (unit + u) * blockDim.x + threadIdx.x, reinterpret_cast<const char*>(row + col) + u * 16);
  unit += units<T>();
}
template <typename T>
__device__ __forceinline__ void take(const uint4* ring, int& unit, bool in, float* f) {
  uint4 v[units<T>()];
#pragma unroll
  for (int u = 0; u < units<T>(); ++u) v[u] = in ? ring[(unit + u) * blockDim.x + threadIdx.x] : make_uint4(0, 0, 0, 0);
  unit += units<T>();
  Pack<T, 8> p;
  static_assert(sizeof(p) == sizeof(v), "");
  memcpy(&p, v, sizeof(p));
  p.get(f);
}

constexpr int kRing = 3;                  // rows fetched ahead
constexpr int kBigD = 4096;               // beyond: 1024 threads, so 64 registers; the sums move to shared memory

// Blocks blockIdx.y = worker; block b of a worker takes its rows b rpb .., then blocks_w rpb further on.  The sums over the
// rows stay in registers (BIG: in shared memory, each thread its own columns) until the end, one partial per block.
// RING: rows are fetched kRing ahead (16-byte pieces only).
template <typename TR, typename TA, int VEC, bool RING, bool BIG>
__global__ void __launch_bounds__(BIG ? 1024 : 512)
blocknorm_backward_kernel(const __grid_constant__ NormArgs a) {
  constexpr int E = 8;
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float s_red[4][32];
  const lsgd_blocknorm_desc& d = a.d;
  const int sub = threadIdx.x / a.tpr;
  const Cols<VEC, E> c{a.tpr, (int)threadIdx.x - sub * a.tpr, d.D};
  const uint32_t w = blockIdx.y;
  const bool has_y = d.y.data != nullptr, pre = d.w_pre.data != nullptr, has_d = d.d_out.data != nullptr;
  const bool token = d.gate_kind == LSGD_GATE_TOKEN, channel = d.gate_kind == LSGD_GATE_CHANNEL;
  float* s_sum = reinterpret_cast<float*>(smem);                        // BIG: [3][8][threads], otherwise [rpb][D] at the end
  uint4* ring = reinterpret_cast<uint4*>(smem + (BIG ? sizeof(float) * 24 * blockDim.x : 0));
  const int stage = ((has_d ? units<TR>() : 0) + (pre ? units<TR>() + units<TA>() : 0) + (has_y ? units<TA>() : 0) +
                     (token ? units<TA>() : 0)) * (int)blockDim.x;
  float wpre[E], wpost[E], ga[E];
  float sum_pre[E], sum_post[E], sum_gate[E];
#pragma unroll
  for (int k = 0; k < E; ++k) sum_pre[k] = sum_post[k] = sum_gate[k] = 0.f;
  const auto add_sum = [&](float (&reg)[E], int which, const float (&x)[E], const float (&y)[E]) {
#pragma unroll
    for (int k = 0; k < E; ++k) {
      if (BIG) {
        float* p = s_sum + (which * E + k) * blockDim.x + threadIdx.x;
        *p = fmaf(x[k], y[k], *p);
      } else {
        reg[k] = fmaf(x[k], y[k], reg[k]);
      }
    }
  };
  const auto gates = [&] {
    read_vector<VEC, E>(at(d.gate, w), c, ga);
#pragma unroll
    for (int k = 0; k < E; ++k) ga[k] = gate_value(ga[k], d.gate_act);
  };
  if (BIG) {
#pragma unroll
    for (int k = 0; k < 3 * E; ++k) s_sum[k * blockDim.x + threadIdx.x] = 0.f;
  } else {
    if (pre) read_vector<VEC, E>(at(d.w_pre, w), c, wpre);
    if (d.post_norm) read_vector<VEC, E>(at(d.w_post, w), c, wpost);
    if (channel) gates();
  }
  const uint32_t step = a.blocks_w * a.rpb;
  const auto fetch = [&](uint32_t t0, int slot) {
    const uint32_t t = t0 + sub;
    if (t0 < a.T && t < a.T && c.in(0)) {
      uint4* s = ring + slot * stage;
      int unit = 0;
      if (has_d) fetch_ahead<TR>(s, unit, at<const TR>(d.d_out, w, t), c.col(0));
      if (pre) {
        fetch_ahead<TR>(s, unit, at<const TR>(d.out, w, t), c.col(0));
        fetch_ahead<TA>(s, unit, at<const TA>(d.d_h, w, t), c.col(0));
      }
      if (has_y) fetch_ahead<TA>(s, unit, at<const TA>(d.y, w, t), c.col(0));
      if (token) fetch_ahead<TA>(s, unit, at<const TA>(d.gate, w, t), c.col(0));
    }
    copy_commit();                        // an empty group keeps the count
  };
  if (RING) {
#pragma unroll
    for (int q = 0; q < kRing - 1; ++q) fetch(min(a.T, (uint32_t)(blockIdx.x * a.rpb) + q * step), q);
  }
  int phase = 0, slot = 0;
  for (uint32_t t0 = blockIdx.x * a.rpb; t0 < a.T; t0 += step, phase ^= 2) {
    const uint32_t t = t0 + sub;
    const bool live = t < a.T;
    const uint32_t r = w * a.T + t;
    int unit = 0;
    const uint4* src = ring;
    if (RING) {
      const uint64_t ahead = (uint64_t)t0 + (uint64_t)(kRing - 1) * step;
      fetch(ahead < a.T ? (uint32_t)ahead : a.T, slot >= 1 ? slot - 1 : kRing - 1);
      copy_wait<kRing - 1>();
      src = ring + slot * stage;
      slot = slot + 1 == kRing ? 0 : slot + 1;
    }
    const auto read = [&](auto tag, const lsgd_rows& m, float (&f)[E]) {
      using T = decltype(tag);
      if (RING) {
        take<T>(src, unit, live && c.in(0), f);
      } else if (live) {
        read_row<T, VEC, E>(at<const T>(m, w, t), c, f);
      } else {
#pragma unroll
        for (int k = 0; k < E; ++k) f[k] = 0.f;
      }
    };
    float g[E];                           // d_out, then the gradient of x'
#pragma unroll
    for (int k = 0; k < E; ++k) g[k] = 0.f;
    if (has_d) read(TR(), d.d_out, g);
    if (pre) {
      float n[E], up[E];
      read(TR(), d.out, n);
      read(TA(), d.d_h, up);
      const float rs = live ? d.rstd_pre[r] : 0.f;
#pragma unroll
      for (int k = 0; k < E; ++k) n[k] *= rs;
      add_sum(sum_pre, 0, up, n);
      if (BIG) read_vector<VEC, E>(at(d.w_pre, w), c, wpre);
      float q = 0.f;
#pragma unroll
      for (int k = 0; k < E; ++k) {
        up[k] *= wpre[k];
        q = fmaf(up[k], n[k], q);
      }
      q = row_sum(q, a.tpr, s_red[phase]) * a.inv_d;
#pragma unroll
      for (int k = 0; k < E; ++k) g[k] += rs * (up[k] - n[k] * q);
    }
    if (live) {
      float o[E];
#pragma unroll
      for (int k = 0; k < E; ++k) o[k] = has_y ? d.alpha * g[k] : g[k];
      write_row<TR, VEC, E>(at<TR>(d.dx, w, t), c, o);
    }
    if (!has_y) continue;
    float n[E];
    read(TA(), d.y, n);
    float rs = 1.f;
    if (d.post_norm) {
      rs = live ? d.rstd_post[r] : 0.f;
#pragma unroll
      for (int k = 0; k < E; ++k) n[k] *= rs;
      if (BIG) read_vector<VEC, E>(at(d.w_post, w), c, wpost);
    }
#pragma unroll
    for (int k = 0; k < E; ++k) g[k] *= d.beta;
    if (token) {
      float z[E];
      read(TA(), d.gate, z);
#pragma unroll
      for (int k = 0; k < E; ++k) {
        const float av = gate_value(z[k], d.gate_act);
        z[k] = g[k] * (d.post_norm ? n[k] * wpost[k] : n[k]) * gate_slope(av, d.gate_act);
        g[k] *= av;
      }
      if (live) write_row<TA, VEC, E>(at<TA>(d.d_gate, w, t), c, z);
    } else if (channel) {
      if (BIG) gates();
      float u[E];
#pragma unroll
      for (int k = 0; k < E; ++k) u[k] = d.post_norm ? n[k] * wpost[k] : n[k];
      add_sum(sum_gate, 2, g, u);
#pragma unroll
      for (int k = 0; k < E; ++k) g[k] *= ga[k];
    }
    if (d.post_norm) {
      add_sum(sum_post, 1, g, n);
      float q = 0.f;
#pragma unroll
      for (int k = 0; k < E; ++k) {
        g[k] *= wpost[k];
        q = fmaf(g[k], n[k], q);
      }
      q = row_sum(q, a.tpr, s_red[phase + 1]) * a.inv_d;
#pragma unroll
      for (int k = 0; k < E; ++k) g[k] = rs * (g[k] - n[k] * q);
    }
    if (live) write_row<TA, VEC, E>(at<TA>(d.dy, w, t), c, g);
  }
  // one partial row per block for each of the three sums
  float* part = a.part + ((size_t)w * a.blocks_w + blockIdx.x) * 3 * d.D;
  if (RING) copy_wait<0>();
  if (BIG && channel) gates();
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    const bool want = j == 0 ? pre && d.d_w_pre.data : j == 1 ? d.post_norm && d.d_w_post.data : channel && d.d_gate.data;
    if (!want) continue;
    float s[E];
#pragma unroll
    for (int k = 0; k < E; ++k) {
      s[k] = BIG ? s_sum[(j * E + k) * blockDim.x + threadIdx.x] : j == 0 ? sum_pre[k] : j == 1 ? sum_post[k] : sum_gate[k];
      if (j == 2) s[k] *= gate_slope(ga[k], d.gate_act);
    }
    if (!BIG && a.rpb > 1) {              // add the block's rows in order
      __syncthreads();
#pragma unroll
      for (int i = 0; i < E / VEC; ++i)
        if (c.in(i))
          for (int k = 0; k < VEC; ++k) s_sum[sub * d.D + c.col(i) + k] = s[i * VEC + k];
      __syncthreads();
      for (int col = threadIdx.x; col < d.D; col += blockDim.x) {
        float v = 0.f;
        for (int q = 0; q < a.rpb; ++q) v += s_sum[q * d.D + col];
        part[j * (size_t)d.D + col] = v;
      }
    } else {
#pragma unroll
      for (int i = 0; i < E / VEC; ++i)
        if (c.in(i))
          for (int k = 0; k < VEC; ++k) part[j * (size_t)d.D + c.col(i) + k] = s[i * VEC + k];
    }
  }
}

// Adds the blocks' partial rows in order.  Block: 32 columns of one of the three sums of one worker (of all workers where
// they share the vector); 8 warps add a run of rows each, then the runs.
constexpr int kJoinThreads = 256;
__global__ void __launch_bounds__(kJoinThreads)
blocknorm_join_kernel(const __grid_constant__ NormArgs a) {
  pdl_wait();
  const lsgd_blocknorm_desc& d = a.d;
  const int j = blockIdx.y;
  const lsgd_rows& o = j == 0 ? d.d_w_pre : j == 1 ? d.d_w_post : d.d_gate;
  if (!o.data || (j == 0 && !d.w_pre.data) || (j == 1 && !d.post_norm) || (j == 2 && d.gate_kind != LSGD_GATE_CHANNEL)) return;
  const bool shared = d.P > 1 && o.stride == 0;
  if (shared && blockIdx.z > 0) return;
  const uint32_t n = a.blocks_w * (shared ? d.P : 1);
  const float* src = a.part + ((size_t)blockIdx.z * a.blocks_w * 3 + j) * d.D;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  __shared__ float s[8][32];
  float acc = 0.f;
  const uint32_t per = (n + 7) / 8, i1 = min(n, (warp + 1) * per);
  if (col < d.D)
#pragma unroll 8
    for (uint32_t i = warp * per; i < i1; ++i) acc += src[(size_t)i * 3 * d.D + col];
  s[warp][lane] = acc;
  __syncthreads();
  if (warp != 0 || col >= d.D) return;
  float v = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q) v += s[q][lane];
  float* dst = at(o, blockIdx.z) + col;
  *dst = d.accumulate ? *dst + v : v;
}

// ------------------------------------------------------------------------------------------------ host
constexpr int kMaxD = 8192;
constexpr int kRingBytes = 220 * 1024;    // dynamic shared memory of a block at most

lsgd_status check_norm(const lsgd_blocknorm_desc* d, bool backward) {
  if (!d || d->struct_size != sizeof(lsgd_blocknorm_desc)) return LSGD_ERR_INVALID_ARG;
  if (d->P < 1 || d->T < 0 || d->D < 1) return LSGD_ERR_INVALID_ARG;
  if (d->resid_dtype < LSGD_F32 || d->resid_dtype > LSGD_BF16 || d->act_dtype < LSGD_F32 || d->act_dtype > LSGD_BF16)
    return LSGD_ERR_INVALID_ARG;
  if (d->resid_dtype == LSGD_BF16 && d->act_dtype == LSGD_F32) return LSGD_ERR_UNSUPPORTED;
  if (d->D > kMaxD || d->P > 65535) return LSGD_ERR_UNSUPPORTED;
  if (d->T >= (int64_t(1) << 31) / d->P) return LSGD_ERR_TOO_LARGE;
  if (d->gate_kind < LSGD_GATE_NONE || d->gate_kind > LSGD_GATE_TOKEN || d->gate_act < LSGD_GATE_IDENTITY ||
      d->gate_act > LSGD_GATE_TANH)
    return LSGD_ERR_INVALID_ARG;
  if (!(d->eps > 0.f) || !(d->eps < 1e30f) || !(d->alpha - d->alpha == 0.f) || !(d->beta - d->beta == 0.f)) return LSGD_ERR_INVALID_ARG;
  const bool has_y = d->y.data != nullptr, pre = d->w_pre.data != nullptr, rows = d->T > 0;
  const bool gated = d->gate_kind != LSGD_GATE_NONE, channel = d->gate_kind == LSGD_GATE_CHANNEL;
  if (!has_y && rows && (d->post_norm || gated || !pre)) return LSGD_ERR_INVALID_ARG;
  const int rb = elem_bytes(d->resid_dtype), ab = elem_bytes(d->act_dtype);
  const int64_t P = d->P, T = d->T, D = d->D;
  if (d->post_norm && (!d->w_post.data || (rows && !d->rstd_post))) return LSGD_ERR_INVALID_ARG;
  if (pre && rows && !d->rstd_pre) return LSGD_ERR_INVALID_ARG;
  if (gated && (rows || channel) && !d->gate.data) return LSGD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(d->rstd_post) | reinterpret_cast<uintptr_t>(d->rstd_pre)) % 4) return LSGD_ERR_ALIGNMENT;
  lsgd_status st;
#define LSGD_ROWS(r, t, bytes, written, shared)                                                   \
  do {                                                                                            \
    if ((r).data && (st = check_rows(r, P, t, D, bytes, written, shared)) != LSGD_OK) return st;  \
  } while (0)
  LSGD_ROWS(d->y, T, ab, false, false);
  LSGD_ROWS(d->gate, channel ? 1 : T, channel ? 4 : ab, false, false);
  LSGD_ROWS(d->w_post, 1, 4, false, false);
  LSGD_ROWS(d->w_pre, 1, 4, false, false);
  LSGD_ROWS(d->out, T, rb, !backward, false);
  if (!backward) {
    if (rows && (!d->x.data || (has_y && !d->out.data) || (pre && !d->h.data))) return LSGD_ERR_INVALID_ARG;
    LSGD_ROWS(d->x, T, rb, false, false);
    LSGD_ROWS(d->h, T, ab, true, false);
    return LSGD_OK;
  }
  if (rows && ((pre && (!d->out.data || !d->d_h.data)) || (!pre && !d->d_out.data) || !d->dx.data || (has_y && !d->dy.data)))
    return LSGD_ERR_INVALID_ARG;
  if (rows && d->gate_kind == LSGD_GATE_TOKEN && !d->d_gate.data) return LSGD_ERR_INVALID_ARG;
  LSGD_ROWS(d->d_out, T, rb, false, false);
  LSGD_ROWS(d->d_h, T, ab, false, false);
  LSGD_ROWS(d->dx, T, rb, true, false);
  LSGD_ROWS(d->dy, T, ab, true, false);
  LSGD_ROWS(d->d_gate, channel ? 1 : T, channel ? 4 : ab, true, channel);
  LSGD_ROWS(d->d_w_post, 1, 4, true, true);
  LSGD_ROWS(d->d_w_pre, 1, 4, true, true);
#undef LSGD_ROWS
  return LSGD_OK;
}

struct Shape {
  int vec, tpr, rpb, threads;
  bool big, ring;
  size_t smem;               // of the backward kernel
};

Shape shape_of(const lsgd_blocknorm_desc* d, bool backward) {
  const int rb = elem_bytes(d->resid_dtype), ab = elem_bytes(d->act_dtype);
  const bool token = d->gate_kind == LSGD_GATE_TOKEN, pre = d->w_pre.data != nullptr;
  Shape s{};
  s.vec = 8;
  auto see = [&](const lsgd_rows& r, int bytes) { s.vec = min_vec(s.vec, row_vec(r, d->P, d->T, d->D, bytes)); };
  see(d->y, ab);
  if (token) see(d->gate, ab);
  see(d->out, rb);
  if (backward) {
    see(d->d_out, rb);
    see(d->d_h, ab);
    see(d->dx, rb);
    see(d->dy, ab);
    if (token) see(d->d_gate, ab);
  } else {
    see(d->x, rb);
    see(d->h, ab);
  }
  const int need = (d->D + 7) / 8;
  s.tpr = 8;
  while (s.tpr < 32 && s.tpr < need) s.tpr *= 2;
  if (need > 32) s.tpr = (need + 31) / 32 * 32;
  s.rpb = s.tpr >= 128 ? 1 : 128 / s.tpr;
  s.threads = s.tpr * s.rpb;
  s.big = d->D > kBigD;
  if (backward) {
    const size_t values = (d->d_out.data ? rb : 0) + (pre ? rb + ab : 0) + (d->y.data ? ab : 0) + (token ? ab : 0);
    const size_t ring = kRing * values * 8 * s.threads;
    const size_t sums = s.big ? sizeof(float) * 24 * s.threads : s.rpb > 1 ? sizeof(float) * (size_t)s.rpb * d->D : 0;
    s.ring = s.vec == 8 && (s.big ? ring + sums : ring) <= kRingBytes;
    s.smem = !s.ring ? sums : s.big ? ring + sums : ring > sums ? ring : sums;
  }
  return s;
}

uint32_t backward_blocks(const lsgd_blocknorm_desc* d, const Shape& s) {
  const int64_t groups = (d->T + s.rpb - 1) / s.rpb;
  const int per_sm = s.threads >= 512 ? 1 : 512 / s.threads;     // what the registers hold at once
  const int64_t n = ((int64_t)sm_count() * per_sm + d->P - 1) / d->P;
  return (uint32_t)(groups < n ? groups : n);
}

template <typename TR, typename TA, int VEC, bool RING, bool BIG>
cudaError_t launch_backward(const NormArgs& a, const Shape& s, cudaStream_t st) {
  static OncePerDevice once;
  if (!once.here()) {
    const cudaError_t e = cudaFuncSetAttribute(blocknorm_backward_kernel<TR, TA, VEC, RING, BIG>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes);
    if (e != cudaSuccess) return e;
    once.here() = true;
  }
  return launch_pdl(blocknorm_backward_kernel<TR, TA, VEC, RING, BIG>, dim3(a.blocks_w, a.d.P), dim3(s.threads), s.smem, st, a);
}

template <typename TR, typename TA, int VEC>
cudaError_t launch(const NormArgs& a, const Shape& s, bool backward, cudaStream_t st) {
  if (!backward)
    return launch_pdl(blocknorm_forward_kernel<TR, TA, VEC>, dim3((a.rows_n + s.rpb - 1) / s.rpb), dim3(s.threads), 0, st, a);
  if (VEC == 8 && s.ring)
    return s.big ? launch_backward<TR, TA, VEC, VEC == 8, true>(a, s, st) : launch_backward<TR, TA, VEC, VEC == 8, false>(a, s, st);
  return s.big ? launch_backward<TR, TA, VEC, false, true>(a, s, st) : launch_backward<TR, TA, VEC, false, false>(a, s, st);
}

template <typename TR, typename TA>
cudaError_t dispatch(const NormArgs& a, const Shape& s, bool backward, cudaStream_t st) {
  return s.vec == 8 ? launch<TR, TA, 8>(a, s, backward, st)
         : s.vec == 2 ? launch<TR, TA, 2>(a, s, backward, st) : launch<TR, TA, 1>(a, s, backward, st);
}

cudaError_t blocknorm(const lsgd_blocknorm_desc* d, bool backward, cudaStream_t st) {
  const Shape s = shape_of(d, backward);
  NormArgs a{};
  a.d = *d;
  a.T = (uint32_t)d->T;
  a.rows_n = (uint32_t)(d->T * d->P);
  a.tpr = s.tpr;
  a.rpb = s.rpb;
  a.inv_d = 1.f / (float)d->D;
  if (backward) {
    a.blocks_w = backward_blocks(d, s);
    a.part = static_cast<float*>(d->scratch);
  }
  cudaError_t e = cudaSuccess;
  if (d->T > 0)
    e = d->resid_dtype == LSGD_BF16 ? dispatch<bf16, bf16>(a, s, backward, st)
        : d->act_dtype == LSGD_BF16 ? dispatch<float, bf16>(a, s, backward, st) : dispatch<float, float>(a, s, backward, st);
  if (e != cudaSuccess || !backward) return e;
  const bool sums = (d->w_pre.data && d->d_w_pre.data) || (d->post_norm && d->d_w_post.data) ||
                    (d->gate_kind == LSGD_GATE_CHANNEL && d->d_gate.data);
  if (!sums) return cudaSuccess;
  return launch_pdl(blocknorm_join_kernel, dim3((d->D + 31) / 32, 3, d->P), dim3(kJoinThreads), 0, st, a);
}

}  // namespace
}  // namespace lsgd

extern "C" {

uint64_t lsgd_blocknorm_scratch_bytes(const lsgd_blocknorm_desc* d) {
  using namespace lsgd;
  if (!d || d->struct_size != sizeof(lsgd_blocknorm_desc) || d->P < 1 || d->T < 0 || d->D < 1 || d->D > kMaxD) return 0;
  return sizeof(float) * 3 * (uint64_t)d->D * d->P * backward_blocks(d, shape_of(d, true));
}

lsgd_status lsgd_blocknorm_forward(const lsgd_blocknorm_desc* d, void* stream) {
  using namespace lsgd;
  const lsgd_status st = check_norm(d, false);
  if (st != LSGD_OK) return st;
  return blocknorm(d, false, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

lsgd_status lsgd_blocknorm_backward(const lsgd_blocknorm_desc* d, void* stream) {
  using namespace lsgd;
  const lsgd_status st = check_norm(d, true);
  if (st != LSGD_OK) return st;
  const uint64_t need = lsgd_blocknorm_scratch_bytes(d);
  if (need && (!d->scratch || d->scratch_bytes < need)) return LSGD_ERR_INVALID_ARG;
  if (need && reinterpret_cast<uintptr_t>(d->scratch) % 256) return LSGD_ERR_ALIGNMENT;
  return blocknorm(d, true, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

}  // extern "C"
