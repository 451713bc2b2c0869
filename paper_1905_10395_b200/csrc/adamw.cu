// AdamW over many tensors in one launch, moments in 32 or in 8 bits.
//
//     m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory: per parameter 4 + 4 bytes of p, 4 or 2 of g, 2 of the copy and 16 bytes (fp32 moments) or 4 (8-bit ones)
// of state.  A warp owns a block of 256 values, 8 a lane, so that the scales of the 8-bit moments (the largest magnitude of a
// block) are one warp reduction and nothing is read twice.  The tensors are cut into chunks of 16 blocks; a persistent grid
// walks the table of chunks (the next one's entry is on its way while one is computed), so tensors of every size are one
// launch.
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
// Blocks on an SM.  8-bit moments: 288 us with two, 266 with three or four (32 classifiers, read out as well).  fp32 moments,
// four long streams more: 146 us with three, 139 with two for 890 MB.
constexpr int kBlocksBytes = 3, kBlocksF32 = 2;

struct Counter {                          // steps taken; the running powers of beta1 and beta2
  double b1t, b2t;
  int64_t t;
  uint32_t done;                          // blocks of the running launch that have ended
};
struct Chunk {                            // 4096 values of a tensor, or what is left of it
  float* p;
  const void* g;
  uint16_t* copy;
  uint32_t block;                         // of the moments, the chunk's first
  int32_t n;                              // values
  float wd;
  int32_t wide;                           // every pointer is aligned to 8 of its values
};
constexpr int kChunkWords = sizeof(Chunk) / 4;

struct StepArgs {
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
// 2^-100: blocks below it are stored as zeros, since the least code (2^-33 of a scale) has to be a number and a reciprocal of
// the scale finite.  What m / sqrt(v) loses with them, sqrt(v) < 2^-50, eps replaces.
constexpr float kTiny = 7.8886091e-31f;
constexpr double kLeastEps8 = 8.8817841970012523e-16;   // 2^-50

__host__ __device__ constexpr float pow2(int e) {
  float r = 1.f;
  for (int i = 0; i < (e < 0 ? -e : e); ++i) r *= e < 0 ? 0.5f : 2.f;
  return r;
}
constexpr int kShiftM = 112, kShiftV = 96;

// Random bits of a number: the multipliers and the first two shifts of the final mixing of xxHash (Y. Collet, 32-bit variant).
__device__ __forceinline__ uint32_t mix(uint32_t h) {
  h *= 0x9E3779B1u;
  h ^= h >> 15;
  h *= 0x85EBCA77u;
  return h ^ (h >> 13);
}

// Codes lie at the top of a word (byte 3) on their way: there they are 4 bits away from the float's bits.
template <int K>
__device__ __forceinline__ uint32_t top_byte(uint32_t w) { return __byte_perm(w, 0, 0x0444 | K << 12); }

// 8 codes times their scale.  2^s scale is one factor where it is finite (FOLD): the same product, rounded once.
template <bool SIGNED, bool FOLD>
__device__ __forceinline__ void decode8(uint2 c, float scale, float2 (&f)[4]) {
  constexpr float kPow = pow2(SIGNED ? kShiftM : kShiftV);
  const float factor = FOLD ? __fmul_rn(scale, kPow) : scale;
  uint32_t w[8] = {top_byte<0>(c.x), top_byte<1>(c.x), top_byte<2>(c.x), top_byte<3>(c.x),
                   top_byte<0>(c.y), top_byte<1>(c.y), top_byte<2>(c.y), top_byte<3>(c.y)};
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    uint32_t bits = w[k] >> 4;
    if (SIGNED) bits = (bits & 0x07F00000u) | (w[k] & 0x80000000u);
    (k & 1 ? f[k >> 1].y : f[k >> 1].x) = __uint_as_float(bits);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (!FOLD) f[k] = mul2(f[k], both(kPow));
    f[k] = mul2(f[k], both(factor));
  }
}
// Scales below this are folded into the powers of two, up and (as reciprocals) down, without overflow or loss.
constexpr float kFoldBelow = 16384.f;

// Scale of a block from its largest magnitude: NaN if that is not finite (top - top), so the whole block reads as NaN.
__device__ __forceinline__ float block_scale(uint32_t top_bits) {
  const float top = __uint_as_float(top_bits);
  return top < kTiny ? 0.f : __fmaf_rn(top, kTop, top - top);
}
// 8 values as codes.  rnd: their hashes; the low half rounds m, the high half v.  The sum of a value's bits and 16 random ones
// below the code is formed 4 bits to the left, so that the code is byte 3 and a sign has left the word.  No code overflows:
// the largest value is at most 4 units in its last place above 1.875, and 15 and the largest random number do not carry.
template <bool SIGNED, bool FOLD>
__device__ __forceinline__ uint2 encode8(const float2 (&z)[4], float scale, const uint32_t (&rnd)[8]) {
  constexpr float kPow = pow2(SIGNED ? -kShiftM : -kShiftV);
  float inv = scale > 0.f ? __frcp_rn(scale) : 0.f;
  const uint32_t least = inv > 0.f ? 0x00100000u : 0u;         // code 1
  if (FOLD) inv = __fmul_rn(inv, kPow);
  uint32_t w[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float2 q = mul2(z[k], both(inv));
    if (!FOLD) q = mul2(q, both(kPow));
    w[2 * k] = __float_as_uint(q.x);
    w[2 * k + 1] = __float_as_uint(q.y);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    // a second moment that is not zero keeps a denominator, also where it is so far below the block's that w is 0
    if (!SIGNED && (k & 1 ? z[k >> 1].y : z[k >> 1].x) > 0.f) w[k] = max(w[k], least);
    w[k] = (w[k] << 4) + __byte_perm(rnd[k], 0, SIGNED ? 0x4104 : 0x4324);
    if (SIGNED) w[k] = (w[k] & 0x7FFFFFFFu) | (__float_as_uint(k & 1 ? z[k >> 1].y : z[k >> 1].x) & 0x80000000u);
  }
  uint2 c;
  c.x = __byte_perm(__byte_perm(w[0], w[1], 0x0073), __byte_perm(w[2], w[3], 0x0073), 0x5410);
  c.y = __byte_perm(__byte_perm(w[4], w[5], 0x0073), __byte_perm(w[6], w[7], 0x0073), 0x5410);
  return c;
}

// Largest magnitude of a block, as bits (NaN is largest); a whole warp calls it.
__device__ __forceinline__ uint32_t block_top(const float2 (&z)[4]) {
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(fabsf(z[k].x)));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(fabsf(z[k].y)));
  }
  return __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top));
}

// 1 / (sqrt(v) root + eps).  eps is not below 2^-126, so the reciprocal's argument is normal; a subnormal v would count as zero,
// so where its root matters beside eps (LOW) a small v is lifted by 2^64 first and its root lowered by 2^32.
template <bool LOW>
__device__ __forceinline__ float reciprocal_root(float v, float root, float eps) {
  float s, r;
  if (LOW && v < 5.421010862427522e-20f) {                     // 2^-64
    v *= 18446744073709551616.f;
    root *= 2.3283064365386963e-10f;
  }
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(v));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(fmaf(s, root, eps)));
  return r;
}
// A root that is taken as zero is below 2^-63, and root is at most 1 / sqrt(1 - beta2) (the first step's): from this eps on
// it is below 2^-22 eps, as the approximations are.
bool low_eps(const lsgd_adamw_desc& d) { return d.eps * std::sqrt(1.0 - d.beta2) < 4.547473508864641e-13; }   // 2^-41

// A sum of products that are rounded first: as a pair the addition would be fused with one of them.
__device__ __forceinline__ float2 sum(float2 a, float2 b) { return make_float2(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y)); }

struct Scalars {
  float step, root, gs;
  uint32_t key;
};

// A lane's 8 values of a block as they lie in memory.
template <typename TG, bool BYTES>
struct Lane8 {
  Pack<float, 8> p;
  Pack<TG, 8> g;
  uint2 cm, cv;
  float sm, sv;
  Pack<float, 8> m, v;
  __device__ __forceinline__ void load(const StepArgs& a, const Chunk& c, int j0, uint32_t block, int lane) {
    p.load(c.p + j0);
    g.load(static_cast<const TG*>(c.g) + j0);
    load_moments(a, block, lane);
  }
  __device__ __forceinline__ void load_moments(const StepArgs& a, uint32_t block, int lane) {
    const size_t s0 = (size_t)block * kBlock + lane * 8;
    if (BYTES) {
      cm = *reinterpret_cast<const uint2*>(static_cast<uint8_t*>(a.m) + s0);
      cv = *reinterpret_cast<const uint2*>(static_cast<uint8_t*>(a.v) + s0);
      sm = a.m_scale[block];
      sv = a.v_scale[block];
    } else {
      m.load(static_cast<float*>(a.m) + s0);
      v.load(static_cast<float*>(a.v) + s0);
    }
  }
};

template <bool SIGNED>
__device__ __forceinline__ void decode_block(uint2 c, float scale, float2 (&f)[4]) {
  if (scale < kFoldBelow) decode8<SIGNED, true>(c, scale, f);
  else decode8<SIGNED, false>(c, scale, f);
}
template <bool SIGNED>
__device__ __forceinline__ uint2 encode_block(const float2 (&z)[4], float scale, const uint32_t (&rnd)[8]) {
  return scale < kFoldBelow ? encode8<SIGNED, true>(z, scale, rnd) : encode8<SIGNED, false>(z, scale, rnd);
}

// The step of 8 values of one block in each lane (32 classifiers of 1.86 million parameters, bf16 gradients, 8-bit moments, bf16
// copies: 163 us for 954 MB, 5.9 TB/s or 0.89 of the measured copy bandwidth; with scalar arithmetic and codes taken apart bit
// by bit it was bound by issue slots, 296 us); `have` of them are the tensor's.
template <typename TG, bool BYTES, bool LOW>
__device__ __forceinline__ void step8(const StepArgs& a, const Scalars& k_, const Chunk& c, const Lane8<TG, BYTES>& in, int j0, uint32_t block,
                                      int lane, int have, bool wide) {
  float2 p[4], g[4], m[4], v[4];
  in.p.get(reinterpret_cast<float*>(p));
  in.g.get(reinterpret_cast<float*>(g));
  if (a.grad_scale) {
#pragma unroll
    for (int k = 0; k < 4; ++k) g[k] = mul2(g[k], both(k_.gs));
  }
  if (BYTES) {
    decode_block<true>(in.cm, in.sm, m);
    decode_block<false>(in.cv, in.sv, v);
  } else {
    in.m.get(reinterpret_cast<float*>(m));
    in.v.get(reinterpret_cast<float*>(v));
  }
  const float decay = -(float)a.lr * c.wd;
#pragma unroll
  for (int k = 0; k < 4; ++k) {           // every product and sum rounded by itself: the moments' bits do not depend on the code
    m[k] = sum(mul2(m[k], both(a.b1)), mul2(g[k], both(a.omb1)));
    v[k] = sum(mul2(v[k], both(a.b2)), mul2(mul2(g[k], both(a.omb2)), g[k]));
    const float2 r = make_float2(reciprocal_root<LOW>(v[k].x, k_.root, a.eps), reciprocal_root<LOW>(v[k].y, k_.root, a.eps));
    p[k] = fma2(mul2(m[k], r), both(-k_.step), fma2(p[k], both(decay), p[k]));   // two roundings of p's size
  }
  if (wide) {
    Pack<float, 8> pp;
    pp.set(reinterpret_cast<const float*>(p));
    pp.store(c.p + j0);
    if (c.copy) {
      Pack<__nv_bfloat16, 8> pc;
      pc.set(reinterpret_cast<const float*>(p));
      pc.store(reinterpret_cast<__nv_bfloat16*>(c.copy) + j0);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float x = k & 1 ? p[k >> 1].y : p[k >> 1].x;
      if (k < have) {
        c.p[j0 + k] = x;
        if (c.copy) reinterpret_cast<__nv_bfloat16*>(c.copy)[j0 + k] = __float2bfloat16_rn(x);
      }
    }
  }
  const size_t s0 = (size_t)block * kBlock + lane * 8;
  if (BYTES) {
    if (have < 8) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k >= have) (k & 1 ? m[k >> 1].y : m[k >> 1].x) = (k & 1 ? v[k >> 1].y : v[k >> 1].x) = 0.f;
    }
    const float sm = block_scale(block_top(m)), sv = block_scale(block_top(v));
    uint32_t rnd[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) rnd[k] = mix(((uint32_t)s0 + k) ^ k_.key);
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.m) + s0) = encode_block<true>(m, sm, rnd);
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.v) + s0) = encode_block<false>(v, sv, rnd);
    if (lane == 0) {
      a.m_scale[block] = sm;
      a.v_scale[block] = sv;
    }
  } else if (have == 8) {
    Pack<float, 8> q;
    q.set(reinterpret_cast<const float*>(m));
    q.store(static_cast<float*>(a.m) + s0);
    q.set(reinterpret_cast<const float*>(v));
    q.store(static_cast<float*>(a.v) + s0);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < have) {
        static_cast<float*>(a.m)[s0 + k] = k & 1 ? m[k >> 1].y : m[k >> 1].x;
        static_cast<float*>(a.v)[s0 + k] = k & 1 ? v[k >> 1].y : v[k >> 1].x;
      }
  }
}

template <typename TG, bool BYTES, bool LOW>
__global__ void __launch_bounds__(kWarps * 32, BYTES ? kBlocksBytes : kBlocksF32)
adamw_step_kernel(const __grid_constant__ StepArgs a) {
  pdl_wait();
  __shared__ Scalars s_k;
  __shared__ __align__(16) uint32_t s_chunk[2][kChunkWords];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const auto chunk_word = [&](uint32_t i) {
    return i < a.n_chunks && threadIdx.x < kChunkWords ? reinterpret_cast<const uint32_t*>(a.chunks + i)[threadIdx.x] : 0;
  };
  const uint32_t word = chunk_word(blockIdx.x);
  if (threadIdx.x < kChunkWords) s_chunk[0][threadIdx.x] = word;
  if (threadIdx.x == 32) {
    const double c1 = 1.0 - a.counter->b1t * a.beta1, c2 = 1.0 - a.counter->b2t * a.beta2;
    s_k.step = (float)(a.lr / c1);
    s_k.root = (float)(1.0 / sqrt(c2));
    s_k.key = mix(mix(a.seed) ^ (uint32_t)(a.counter->t + 1));
    s_k.gs = a.grad_scale ? *a.grad_scale : 1.f;
  }
  __syncthreads();
  const Scalars k = s_k;
  int turn = 0;
  for (uint32_t i = blockIdx.x; i < a.n_chunks; i += gridDim.x) {
    const uint32_t next = chunk_word(i + gridDim.x);           // i + gridDim.x < 2^32: there are less than 2^31 chunks
    const Chunk& c = *reinterpret_cast<const Chunk*>(s_chunk[turn]);
    if (c.wide && c.n == kChunk) {
      Lane8<TG, BYTES> in[2];
      constexpr int kAhead = BYTES ? 2 : 1;                    // blocks whose loads are in flight before the first is computed
#pragma unroll
      for (int h = 0; h < 2; h += kAhead) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          const int b = warp + (h + q) * kWarps;
          in[q].load(a, c, b * kBlock + lane * 8, c.block + b, lane);
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          const int b = warp + (h + q) * kWarps;
          step8<TG, BYTES, LOW>(a, k, c, in[q], b * kBlock + lane * 8, c.block + b, lane, 8, true);
        }
      }
    } else {
      for (int b = warp; b * kBlock < c.n; b += kWarps) {      // whole warps
        const int j0 = b * kBlock + lane * 8, have = max(0, min(8, c.n - j0));
        const bool wide = c.wide && have == 8;
        Lane8<TG, BYTES> in;
        if (wide) {
          in.load(a, c, j0, c.block + b, lane);
        } else {
          float f[8], h[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            f[q] = q < have ? c.p[j0 + q] : 0.f;
            h[q] = q < have ? (float)static_cast<const TG*>(c.g)[j0 + q] : 0.f;
          }
          in.p.set(f);
          in.g.set(h);
          in.load_moments(a, c.block + b, lane);
        }
        step8<TG, BYTES, LOW>(a, k, c, in, j0, c.block + b, lane, have, wide);
      }
    }
    turn ^= 1;
    if (threadIdx.x < kChunkWords) s_chunk[turn][threadIdx.x] = next;
    __syncthreads();
  }
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

// A warp reads out kReadBlocks blocks at a time: 100 us for 596 MB, 0.91 of the copy bandwidth.
constexpr int kReadBlocks = 4;
__global__ void __launch_bounds__(256)
adamw_moments_kernel(const uint8_t* m, const uint8_t* v, const float* m_scale, const float* v_scale, float* m_out, float* v_out,
                     uint32_t blocks) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const uint64_t step = (uint64_t)gridDim.x * 8 * kReadBlocks;
  for (uint64_t b0 = ((uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * kReadBlocks; b0 < blocks; b0 += step) {
    uint2 cm[kReadBlocks], cv[kReadBlocks];
    float sm[kReadBlocks], sv[kReadBlocks];
#pragma unroll
    for (int q = 0; q < kReadBlocks; ++q) {
      if (b0 + q >= blocks) break;
      cm[q] = *reinterpret_cast<const uint2*>(m + (b0 + q) * kBlock + lane * 8);
      cv[q] = *reinterpret_cast<const uint2*>(v + (b0 + q) * kBlock + lane * 8);
      sm[q] = m_scale[b0 + q];
      sv[q] = v_scale[b0 + q];
    }
#pragma unroll
    for (int q = 0; q < kReadBlocks; ++q) {
      if (b0 + q >= blocks) break;
      float2 f[4];
      Pack<float, 8> o;
      if (m_out) {
        decode_block<true>(cm[q], sm[q], f);
        o.set(reinterpret_cast<const float*>(f));
        o.store(m_out + (b0 + q) * kBlock + lane * 8);
      }
      if (v_out) {
        decode_block<false>(cv[q], sv[q], f);
        o.set(reinterpret_cast<const float*>(f));
        o.store(v_out + (b0 + q) * kBlock + lane * 8);
      }
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
      !((float)d->eps >= 1.1754944e-38f))
    return LSGD_ERR_INVALID_ARG;
  if (d->state_dtype == LSGD_STATE_8BIT && d->eps < kLeastEps8) return LSGD_ERR_INVALID_ARG;
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
Chunk* chunks_of(const lsgd_adamw_ctx* h) { return reinterpret_cast<Chunk*>(static_cast<char*>(h->slab) + 256); }

template <typename TG, bool BYTES>
cudaError_t launch_step(const StepArgs& a, bool low, cudaStream_t s) {
  const uint32_t cap = (uint32_t)sm_count() * (BYTES ? kBlocksBytes : kBlocksF32);
  const uint32_t grid = a.n_chunks < 1 ? 1 : a.n_chunks < cap ? a.n_chunks : cap;   // one block even with nothing to do: it counts the step
  return low ? launch_pdl(adamw_step_kernel<TG, BYTES, true>, dim3(grid), dim3(kWarps * 32), 0, s, a)
             : launch_pdl(adamw_step_kernel<TG, BYTES, false>, dim3(grid), dim3(kWarps * 32), 0, s, a);
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
  const size_t bytes = 256 + sizeof(Chunk) * (size_t)chunks;
  char* host = new (std::nothrow) char[bytes]();
  if (!host) {
    delete h;
    return LSGD_ERR_CUDA;
  }
  Counter* counter = reinterpret_cast<Counter*>(host);
  counter->b1t = counter->b2t = 1.0;
  Chunk* c = reinterpret_cast<Chunk*>(host + 256);
  const size_t gb = elem_bytes(desc->grad_dtype);
  int64_t at = 0;
  for (int i = 0; i < n; ++i) {
    uint16_t* copy = desc->copies ? desc->copies[i] : nullptr;
    const bool wide = aligned(desc->params[i], 32) && aligned(desc->grads[i], 8 * gb) && aligned(copy, 16);
    for (int64_t j = 0; j < desc->sizes[i]; j += kChunk, ++c) {
      c->p = desc->params[i] + j;
      c->g = static_cast<const char*>(desc->grads[i]) + j * gb;
      c->copy = copy ? copy + j : nullptr;
      c->block = (uint32_t)((at + j) / kBlock);
      c->n = (int32_t)(desc->sizes[i] - j < kChunk ? desc->sizes[i] - j : kChunk);
      c->wd = desc->weight_decay[i];
      c->wide = wide;
    }
    at += padded(desc->sizes[i]);
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
  // ordered before the first step: a blocking copy from pageable memory may return before its last piece has arrived, and
  // nothing orders a non-blocking stream behind the legacy one.  `host` dies here, so the copy is drained.
  ok = ok && cudaMemcpyAsync(h->slab, host, bytes, cudaMemcpyHostToDevice, h->stream) == cudaSuccess;
  ok = ok && cudaStreamSynchronize(h->stream) == cudaSuccess;
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
  const bool bytes = h->d.state_dtype == LSGD_STATE_8BIT, low = low_eps(h->d);
  const cudaError_t e =
      h->d.grad_dtype == LSGD_BF16
          ? (bytes ? launch_step<__nv_bfloat16, true>(a, low, h->stream) : launch_step<__nv_bfloat16, false>(a, low, h->stream))
          : (bytes ? launch_step<float, true>(a, low, h->stream) : launch_step<float, false>(a, low, h->stream));
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
  const uint32_t blocks = (uint32_t)(h->values / kBlock);
  const int64_t want = ((int64_t)blocks + 8 * kReadBlocks - 1) / (8 * kReadBlocks), cap = (int64_t)sm_count() * 8;
  return launch_pdl(adamw_moments_kernel, dim3((unsigned)(want < cap ? want : cap)), dim3(256), 0, h->stream,
                    static_cast<const uint8_t*>(h->d.m), static_cast<const uint8_t*>(h->d.v), h->d.m_scale, h->d.v_scale, m_out,
                    v_out, blocks) == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

lsgd_status lsgd_adamw_get_step(lsgd_adamw_handle h, int64_t* n) {
  using namespace lsgd;
  if (!h || !n) return LSGD_ERR_INVALID_ARG;
  if (!on_own_device(h)) return LSGD_ERR_STATE;
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
  int was = h->device;                    // a NULL stream is that of the current device
  const bool moved = cudaGetDevice(&was) == cudaSuccess && was != h->device && cudaSetDevice(h->device) == cudaSuccess;
  cudaStreamSynchronize(h->stream);
  const cudaError_t e = cudaFree(h->slab);
  if (moved) cudaSetDevice(was);
  delete h;
  return e == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

}  // extern "C"
