// AdamW over many tensors in one launch, moments in 32 or in 8 bits.
//
//     m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory: per parameter 4 + 4 bytes of p, 4 or 2 of g, 2 of the copy and 16 bytes (fp32 moments) or 4 (8-bit ones)
// of state.  A warp owns a block of 256 values, 8 a lane, so that the scales of the 8-bit moments (the largest magnitude of a
// block) are one warp reduction and nothing is read twice.  The tensors are cut into chunks of 16 blocks; a persistent grid
// walks the table of chunks, so tensors of every size are one launch.
//
// An 8-bit code c stands for bits(c << 20) * 2^s * scale: c's bits become exponent and fraction of a small fp32 number
// (exponent field from 0, so the lowest codes are fp32 subnormals, which the hardware multiplies at full speed), and the
// power of two moves it to 0 .. 1.875.  Encoding adds 16 random bits below the code to the same integer and cuts them off:
// rounding up happens with the probability of the part that is cut.
#include <cmath>
#include <new>

#include "lm_ops.h"

struct lsgd_adamw_ctx {
  int device;
  cudaStream_t stream;
  lsgd_adamw_desc d;
  int64_t values;
  uint32_t chunks;
  void* slab;
};

namespace lsgd {
namespace {

constexpr int kBlock = 256;               // values that share a scale
constexpr int kWarps = 8;
constexpr int kChunk = kBlock * 2 * kWarps;

struct Tensor {                           // one entry per tensor, device memory
  float* p;
  const void* g;
  uint16_t* copy;
  int64_t n;                              // values
  int64_t at;                             // first value of its moments
  float wd;
  int32_t wide;                           // every pointer is aligned to 8 of its values
};
struct Counter {                          // steps taken; the running powers of beta1 and beta2
  double b1t, b2t;
  int64_t t;
  uint32_t done;                          // blocks of the running launch that have ended
};
struct Chunk {
  int32_t tensor;
  uint32_t index;                         // of the tensor's chunks
};

struct StepArgs {
  const Tensor* tensors;
  const Chunk* chunks;
  Counter* counter;
  uint32_t n_chunks;
  void *m, *v;
  float *m_scale, *v_scale;
  const float* grad_scale;
  double beta1, beta2, lr;
  float b1, omb1, b2, omb2, eps;
  uint32_t seed;
};

constexpr float kTop = 0.53333336f;       // 1 / 1.875: a block's largest magnitude is code 1.875
constexpr float kTiny = 7.8886091e-31f;   // 2^-100: blocks below it are zero

__host__ __device__ constexpr float pow2(int e) {
  float r = 1.f;
  for (int i = 0; i < (e < 0 ? -e : e); ++i) r *= e < 0 ? 0.5f : 2.f;
  return r;
}
constexpr int kShiftM = 112, kShiftV = 96;

__device__ __forceinline__ uint32_t mix(uint32_t h) {
  h *= 0x9E3779B1u;
  h ^= h >> 15;
  h *= 0x85EBCA77u;
  return h ^ (h >> 13);
}

__device__ __forceinline__ float decode_m(uint32_t c, float scale) {
  const float a = __fmul_rn(__fmul_rn(__uint_as_float((c & 127u) << 20), pow2(kShiftM)), scale);
  return c & 128u ? -a : a;
}
__device__ __forceinline__ float decode_v(uint32_t c, float scale) {
  return __fmul_rn(__fmul_rn(__uint_as_float(c << 20), pow2(kShiftV)), scale);
}
// scale of a block from its largest magnitude, and the reciprocal that codes are made with.  A magnitude that is not finite
// stays in the scale, so the block reads as NaN.
__device__ __forceinline__ float block_scale(uint32_t top_bits, float& inv) {
  const float top = __uint_as_float(top_bits);
  const float scale = top < kTiny ? 0.f : __fmul_rn(top, kTop);
  inv = scale > 0.f ? __frcp_rn(scale) : 0.f;
  return scale;
}
__device__ __forceinline__ uint32_t encode_m(float z, float inv, uint32_t rnd16) {
  const uint32_t bits = __float_as_uint(__fmul_rn(__fmul_rn(fabsf(z), inv), pow2(-kShiftM)));
  const uint32_t c = min((bits + (rnd16 << 4)) >> 20, 127u);
  return c | (z < 0.f ? 128u : 0u);
}
__device__ __forceinline__ uint32_t encode_v(float z, float inv, uint32_t rnd16) {
  const uint32_t bits = __float_as_uint(__fmul_rn(__fmul_rn(z, inv), pow2(-kShiftV)));
  const uint32_t c = min((bits + (rnd16 << 4)) >> 20, 255u);
  return bits ? max(c, 1u) : c;           // a second moment that is not zero keeps a denominator
}

__device__ __forceinline__ float approx_sqrt(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

template <typename TG, bool BYTES>
__global__ void __launch_bounds__(kWarps * 32)
adamw_step_kernel(const __grid_constant__ StepArgs a) {
  pdl_wait();
  __shared__ float s_k[2];
  __shared__ uint32_t s_key;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    const double c1 = 1.0 - a.counter->b1t * a.beta1, c2 = 1.0 - a.counter->b2t * a.beta2;
    s_k[0] = (float)(a.lr / c1);
    s_k[1] = (float)(1.0 / sqrt(c2));
    s_key = mix(mix(a.seed) ^ (uint32_t)(a.counter->t + 1));
  }
  __syncthreads();
  const float step = s_k[0], root = s_k[1];
  const uint32_t key = s_key;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  for (uint32_t i = blockIdx.x; i < a.n_chunks; i += gridDim.x) {
    const Chunk ch = a.chunks[i];
    const Tensor t = a.tensors[ch.tensor];
    const float keep = (float)(1.0 - a.lr * (double)t.wd);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int64_t j0 = (int64_t)ch.index * kChunk + (half * kWarps + warp) * kBlock + lane * 8;
      const int64_t b0 = j0 - lane * 8;
      if (b0 >= t.n) continue;            // whole warp
      const int have = t.n - j0 >= 8 ? 8 : t.n - j0 > 0 ? (int)(t.n - j0) : 0;
      const bool wide = t.wide && have == 8;
      const int64_t s0 = t.at + j0;       // moments
      float p[8], g[8], m[8], v[8];
      if (wide) {
        Pack<float, 8> pp;
        pp.load(t.p + j0);
        pp.get(p);
        Pack<TG, 8> pg;
        pg.load(static_cast<const TG*>(t.g) + j0);
        pg.get(g);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          p[k] = k < have ? t.p[j0 + k] : 0.f;
          g[k] = k < have ? (float)static_cast<const TG*>(t.g)[j0 + k] : 0.f;
        }
      }
      if (a.grad_scale) {
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = __fmul_rn(g[k], gs);
      }
      if (BYTES) {
        const uint2 cm = *reinterpret_cast<const uint2*>(static_cast<uint8_t*>(a.m) + s0);
        const uint2 cv = *reinterpret_cast<const uint2*>(static_cast<uint8_t*>(a.v) + s0);
        const float sm = a.m_scale[s0 / kBlock], sv = a.v_scale[s0 / kBlock];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          m[k] = decode_m((k < 4 ? cm.x : cm.y) >> (8 * (k & 3)) & 255u, sm);
          v[k] = decode_v((k < 4 ? cv.x : cv.y) >> (8 * (k & 3)) & 255u, sv);
        }
      } else {
        Pack<float, 8> q;
        q.load(static_cast<float*>(a.m) + s0);
        q.get(m);
        q.load(static_cast<float*>(a.v) + s0);
        q.get(v);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        m[k] = __fadd_rn(__fmul_rn(m[k], a.b1), __fmul_rn(g[k], a.omb1));
        v[k] = __fadd_rn(__fmul_rn(v[k], a.b2), __fmul_rn(__fmul_rn(g[k], a.omb2), g[k]));
        p[k] = p[k] * keep - step * __fdividef(m[k], fmaf(approx_sqrt(v[k]), root, a.eps));
      }
      if (wide) {
        Pack<float, 8> pp;
        pp.set(p);
        pp.store(t.p + j0);
        if (t.copy) {
          Pack<__nv_bfloat16, 8> pc;
          pc.set(p);
          pc.store(reinterpret_cast<__nv_bfloat16*>(t.copy) + j0);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k < have) {
            t.p[j0 + k] = p[k];
            if (t.copy) reinterpret_cast<__nv_bfloat16*>(t.copy)[j0 + k] = __float2bfloat16_rn(p[k]);
          }
      }
      if (BYTES) {
        uint32_t tm = 0, tv = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (k >= have) m[k] = v[k] = 0.f;
          tm = max(tm, __float_as_uint(m[k]) & 0x7FFFFFFFu);
          tv = max(tv, __float_as_uint(v[k]) & 0x7FFFFFFFu);
        }
        tm = __reduce_max_sync(0xFFFFFFFFu, tm);
        tv = __reduce_max_sync(0xFFFFFFFFu, tv);
        float im, iv;
        const float sm = block_scale(tm, im), sv = block_scale(tv, iv);
        uint32_t wm[2] = {0, 0}, wv[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t h = mix((uint32_t)(s0 + k) ^ key);
          wm[k >> 2] |= encode_m(m[k], im, h & 0xFFFFu) << (8 * (k & 3));
          wv[k >> 2] |= encode_v(v[k], iv, h >> 16) << (8 * (k & 3));
        }
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.m) + s0) = make_uint2(wm[0], wm[1]);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.v) + s0) = make_uint2(wv[0], wv[1]);
        if (lane == 0) {
          a.m_scale[s0 / kBlock] = sm;
          a.v_scale[s0 / kBlock] = sv;
        }
      } else if (have == 8) {
        Pack<float, 8> q;
        q.set(m);
        q.store(static_cast<float*>(a.m) + s0);
        q.set(v);
        q.store(static_cast<float*>(a.v) + s0);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k < have) {
            static_cast<float*>(a.m)[s0 + k] = m[k];
            static_cast<float*>(a.v)[s0 + k] = v[k];
          }
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {                 // every block has read the counter by the time the last one moves it on
    __threadfence();
    if (atomicAdd(&a.counter->done, 1u) == gridDim.x - 1) {
      a.counter->done = 0;
      a.counter->t += 1;
      a.counter->b1t *= a.beta1;
      a.counter->b2t *= a.beta2;
    }
  }
}

__global__ void __launch_bounds__(256)
adamw_moments_kernel(const uint8_t* m, const uint8_t* v, const float* m_scale, const float* v_scale, float* m_out, float* v_out,
                     int64_t values) {
  pdl_wait();
  const int64_t stride = (int64_t)gridDim.x * blockDim.x * 8;
  for (int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * 8; i < values; i += stride) {
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float* out = which ? v_out : m_out;
      if (!out) continue;
      const uint2 c = *reinterpret_cast<const uint2*>((which ? v : m) + i);
      const float s = (which ? v_scale : m_scale)[i / kBlock];
      float f[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t b = (k < 4 ? c.x : c.y) >> (8 * (k & 3)) & 255u;
        f[k] = which ? decode_v(b, s) : decode_m(b, s);
      }
      Pack<float, 8> o;
      o.set(f);
      o.store(out + i);
    }
  }
}

__global__ void adamw_counter_kernel(Counter* c, int64_t t, double b1t, double b2t) {
  pdl_wait();
  c->t = t;
  c->b1t = b1t;
  c->b2t = b2t;
  c->done = 0;
}

int64_t padded(int64_t n) { return (n + kBlock - 1) / kBlock * kBlock; }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool on_own_device(const lsgd_adamw_ctx* h) {
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && dev == h->device;
}

lsgd_status check_adamw(const lsgd_adamw_desc* d) {
  if (!d || d->struct_size != sizeof(lsgd_adamw_desc) || d->n_tensors < 1) return LSGD_ERR_INVALID_ARG;
  if (!d->sizes || !d->params || !d->grads || !d->weight_decay) return LSGD_ERR_INVALID_ARG;
  if (d->grad_dtype < LSGD_F32 || d->grad_dtype > LSGD_BF16 || d->state_dtype < LSGD_STATE_F32 || d->state_dtype > LSGD_STATE_8BIT)
    return LSGD_ERR_INVALID_ARG;
  if (!(d->beta1 >= 0 && d->beta1 < 1) || !(d->beta2 >= 0 && d->beta2 < 1) || !(d->eps > 0) || !std::isfinite((float)d->eps) ||
      !((float)d->eps > 0))
    return LSGD_ERR_INVALID_ARG;
  const int64_t values = lsgd_adamw_state_values(d->n_tensors, d->sizes);
  if (values < 0) return LSGD_ERR_INVALID_ARG;
  if (values / kBlock >= int64_t(1) << 32) return LSGD_ERR_TOO_LARGE;
  const size_t gb = elem_bytes(d->grad_dtype);
  for (int i = 0; i < d->n_tensors; ++i) {
    if (!std::isfinite(d->weight_decay[i])) return LSGD_ERR_INVALID_ARG;
    if (d->sizes[i] == 0) continue;
    if (!d->params[i] || !d->grads[i]) return LSGD_ERR_INVALID_ARG;
    if (!aligned(d->params[i], 4) || !aligned(d->grads[i], gb) || (d->copies && !aligned(d->copies[i], 2))) return LSGD_ERR_ALIGNMENT;
  }
  if (values == 0) return LSGD_OK;
  if (!d->m || !d->v) return LSGD_ERR_INVALID_ARG;
  if (!aligned(d->m, 32) || !aligned(d->v, 32)) return LSGD_ERR_ALIGNMENT;
  if (d->state_dtype == LSGD_STATE_8BIT) {
    if (!d->m_scale || !d->v_scale) return LSGD_ERR_INVALID_ARG;
    if (!aligned(d->m_scale, 4) || !aligned(d->v_scale, 4)) return LSGD_ERR_ALIGNMENT;
  }
  return LSGD_OK;
}

Counter* counter_of(const lsgd_adamw_ctx* h) { return static_cast<Counter*>(h->slab); }
Tensor* tensors_of(const lsgd_adamw_ctx* h) { return reinterpret_cast<Tensor*>(static_cast<char*>(h->slab) + 256); }
Chunk* chunks_of(const lsgd_adamw_ctx* h) { return reinterpret_cast<Chunk*>(tensors_of(h) + h->d.n_tensors); }

template <typename TG, bool BYTES>
cudaError_t launch_step(const StepArgs& a, cudaStream_t s) {
  const uint32_t cap = (uint32_t)sm_count() * 4;
  const uint32_t grid = a.n_chunks < 1 ? 1 : a.n_chunks < cap ? a.n_chunks : cap;   // one block even with nothing to do: it counts the step
  return launch_pdl(adamw_step_kernel<TG, BYTES>, dim3(grid), dim3(kWarps * 32), 0, s, a);
}

}  // namespace
}  // namespace lsgd

extern "C" {

int64_t lsgd_adamw_state_values(int32_t n_tensors, const int64_t* sizes) {
  using namespace lsgd;
  if (n_tensors < 0 || (n_tensors > 0 && !sizes)) return -1;
  int64_t n = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (sizes[i] < 0 || sizes[i] > (int64_t(1) << 48)) return -1;
    n += padded(sizes[i]);
    if (n > int64_t(1) << 50) return -1;
  }
  return n;
}

lsgd_status lsgd_adamw_create(const lsgd_adamw_desc* desc, lsgd_adamw_handle* out) {
  using namespace lsgd;
  if (out) *out = nullptr;
  if (!out) return LSGD_ERR_INVALID_ARG;
  const lsgd_status st = check_adamw(desc);
  if (st != LSGD_OK) return st;
  lsgd_adamw_ctx* h = new (std::nothrow) lsgd_adamw_ctx();
  if (!h) return LSGD_ERR_CUDA;
  h->d = *desc;
  h->stream = static_cast<cudaStream_t>(desc->stream);
  if (cudaGetDevice(&h->device) != cudaSuccess) {
    delete h;
    return LSGD_ERR_CUDA;
  }
  const int n = desc->n_tensors;
  uint64_t chunks = 0;
  for (int i = 0; i < n; ++i) chunks += (uint64_t)((desc->sizes[i] + kChunk - 1) / kChunk);
  const size_t bytes = 256 + sizeof(Tensor) * (size_t)n + sizeof(Chunk) * (size_t)chunks;
  char* host = new (std::nothrow) char[bytes]();
  if (!host) {
    delete h;
    return LSGD_ERR_CUDA;
  }
  Counter* counter = reinterpret_cast<Counter*>(host);
  counter->b1t = counter->b2t = 1.0;
  Tensor* t = reinterpret_cast<Tensor*>(host + 256);
  Chunk* c = reinterpret_cast<Chunk*>(t + n);
  const size_t gb = elem_bytes(desc->grad_dtype);
  int64_t at = 0;
  for (int i = 0; i < n; ++i) {
    t[i].p = desc->params[i];
    t[i].g = desc->grads[i];
    t[i].copy = desc->copies ? desc->copies[i] : nullptr;
    t[i].n = desc->sizes[i];
    t[i].at = at;
    t[i].wd = desc->weight_decay[i];
    t[i].wide = aligned(t[i].p, 32) && aligned(t[i].g, 8 * gb) && aligned(t[i].copy, 16);
    at += padded(t[i].n);
    const uint64_t k = (uint64_t)((t[i].n + kChunk - 1) / kChunk);
    for (uint64_t q = 0; q < k; ++q) *c++ = Chunk{i, (uint32_t)q};
  }
  h->values = at;
  h->chunks = (uint32_t)chunks;
  h->d.sizes = nullptr;
  h->d.params = nullptr;
  h->d.grads = nullptr;
  h->d.copies = nullptr;
  h->d.weight_decay = nullptr;
  bool ok = cudaMalloc(&h->slab, bytes) == cudaSuccess;
  if (!ok) h->slab = nullptr;
  ok = ok && cudaMemcpy(h->slab, host, bytes, cudaMemcpyHostToDevice) == cudaSuccess;
  delete[] host;
  if (!ok) {
    if (h->slab) cudaFree(h->slab);
    delete h;
    return LSGD_ERR_CUDA;
  }
  *out = h;
  return LSGD_OK;
}

lsgd_status lsgd_adamw_step(lsgd_adamw_handle h, double lr, const float* grad_scale) {
  using namespace lsgd;
  if (!h || !std::isfinite(lr) || lr < 0) return LSGD_ERR_INVALID_ARG;
  if (!aligned(grad_scale, 4)) return LSGD_ERR_ALIGNMENT;
  if (!on_own_device(h)) return LSGD_ERR_STATE;
  StepArgs a{};
  a.tensors = tensors_of(h);
  a.chunks = chunks_of(h);
  a.counter = counter_of(h);
  a.n_chunks = h->chunks;
  a.m = h->d.m;
  a.v = h->d.v;
  a.m_scale = h->d.m_scale;
  a.v_scale = h->d.v_scale;
  a.grad_scale = grad_scale;
  a.beta1 = h->d.beta1;
  a.beta2 = h->d.beta2;
  a.lr = lr;
  a.b1 = (float)h->d.beta1;
  a.omb1 = (float)(1.0 - h->d.beta1);
  a.b2 = (float)h->d.beta2;
  a.omb2 = (float)(1.0 - h->d.beta2);
  a.eps = (float)h->d.eps;
  a.seed = h->d.seed;
  const bool bytes = h->d.state_dtype == LSGD_STATE_8BIT;
  const cudaError_t e = h->d.grad_dtype == LSGD_BF16
                            ? (bytes ? launch_step<__nv_bfloat16, true>(a, h->stream) : launch_step<__nv_bfloat16, false>(a, h->stream))
                            : (bytes ? launch_step<float, true>(a, h->stream) : launch_step<float, false>(a, h->stream));
  return e == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

lsgd_status lsgd_adamw_moments(lsgd_adamw_handle h, float* m_out, float* v_out) {
  using namespace lsgd;
  if (!h) return LSGD_ERR_INVALID_ARG;
  if (!aligned(m_out, 32) || !aligned(v_out, 32)) return LSGD_ERR_ALIGNMENT;
  if (!on_own_device(h)) return LSGD_ERR_STATE;
  if (h->values == 0 || (!m_out && !v_out)) return LSGD_OK;
  if (h->d.state_dtype == LSGD_STATE_F32) {
    const size_t n = sizeof(float) * (size_t)h->values;
    if (m_out && cudaMemcpyAsync(m_out, h->d.m, n, cudaMemcpyDeviceToDevice, h->stream) != cudaSuccess) return LSGD_ERR_CUDA;
    if (v_out && cudaMemcpyAsync(v_out, h->d.v, n, cudaMemcpyDeviceToDevice, h->stream) != cudaSuccess) return LSGD_ERR_CUDA;
    return LSGD_OK;
  }
  const int64_t blocks = (h->values / 8 + 255) / 256, cap = (int64_t)sm_count() * 8;
  return launch_pdl(adamw_moments_kernel, dim3((unsigned)(blocks < cap ? blocks : cap)), dim3(256), 0, h->stream,
                    static_cast<const uint8_t*>(h->d.m), static_cast<const uint8_t*>(h->d.v), h->d.m_scale, h->d.v_scale, m_out,
                    v_out, h->values) == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

lsgd_status lsgd_adamw_get_step(lsgd_adamw_handle h, int64_t* n) {
  using namespace lsgd;
  if (!h || !n) return LSGD_ERR_INVALID_ARG;
  Counter c{};
  if (cudaMemcpyAsync(&c, h->slab, sizeof(c), cudaMemcpyDeviceToHost, h->stream) != cudaSuccess) return LSGD_ERR_CUDA;
  if (cudaStreamSynchronize(h->stream) != cudaSuccess) return LSGD_ERR_CUDA;
  *n = c.t;
  return LSGD_OK;
}

lsgd_status lsgd_adamw_set_step(lsgd_adamw_handle h, int64_t n) {
  using namespace lsgd;
  if (!h || n < 0 || n >= int64_t(1) << 31) return LSGD_ERR_INVALID_ARG;
  if (!on_own_device(h)) return LSGD_ERR_STATE;
  return launch_pdl(adamw_counter_kernel, dim3(1), dim3(1), 0, h->stream, counter_of(h), n, std::pow(h->d.beta1, (double)n),
                    std::pow(h->d.beta2, (double)n)) == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

lsgd_status lsgd_adamw_destroy(lsgd_adamw_handle h) {
  if (!h) return LSGD_OK;
  cudaStreamSynchronize(h->stream);
  const cudaError_t e = cudaFree(h->slab);
  delete h;
  return e == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

}  // extern "C"
