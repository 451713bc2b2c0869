// Shared by the operators of a language model's training step (embed.cu, blocknorm.cu, adamw.cu): typed row access of
// 8, 2 or 1 values and the host's checks of lsgd_rows.
#pragma once
#include <cuda_bf16.h>

#include "internal.h"

namespace lsgd {

inline int elem_bytes(int dtype) { return dtype == LSGD_BF16 ? 2 : 4; }

// A device copy of lsgd_rows whose row index runs over all workers' rows.
template <typename T>
struct Rows {
  T* p;
  int64_t ld, stride;
  __device__ __forceinline__ T* row(uint32_t worker, uint32_t t) const { return p + worker * stride + t * ld; }
};
template <typename T>
inline Rows<T> rows_of(const lsgd_rows& r) {
  return Rows<T>{static_cast<T*>(r.data), r.ld, r.stride};
}

// Host: a matrix of P x T rows of D values can be addressed (strides not negative, offsets within 63 bits), is aligned
// to its element, and, if it is written, does not overlap itself.
inline lsgd_status check_rows(const lsgd_rows& r, int64_t P, int64_t T, int64_t D, int bytes, bool written,
                              bool shared_ok = false) {
  if (r.ld < 0 || r.stride < 0) return LSGD_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(r.data) % bytes) return LSGD_ERR_ALIGNMENT;
  const int64_t lim = int64_t(1) << 56;
  if ((T > 1 && r.ld > lim / T) || (P > 1 && r.stride > lim / P)) return LSGD_ERR_TOO_LARGE;
  if (written && T > 0) {
    const bool many_t = T > 1, many_p = P > 1 && !(shared_ok && r.stride == 0);
    if (many_t && r.ld < D) return LSGD_ERR_INVALID_ARG;
    if (many_p) {
      const bool worker_major = r.stride >= (many_t ? (T - 1) * r.ld : 0) + D;
      const bool row_major = r.stride >= D && (!many_t || r.ld >= (P - 1) * r.stride + D);
      if (!worker_major && !row_major) return LSGD_ERR_INVALID_ARG;
    }
  }
  return LSGD_OK;
}

// Widest piece (8, 2 or 1 values) that every row of the matrix can be moved in.
inline int row_vec(const lsgd_rows& r, int64_t P, int64_t T, int64_t D, int bytes) {
  if (!r.data) return 8;
  auto fits = [&](int vec, int align) {
    return D % vec == 0 && reinterpret_cast<uintptr_t>(r.data) % align == 0 && (T <= 1 || (r.ld * bytes) % align == 0) &&
           (P <= 1 || (r.stride * bytes) % align == 0);
  };
  if (fits(8, 8 * bytes)) return 8;
  if (fits(2, 2 * bytes)) return 2;
  return 1;
}
inline int min_vec(int a, int b) { return a < b ? a : b; }

#if defined(__CUDACC__)
// VEC values of type T as they lie in memory (raw registers), and as fp32.
template <typename T, int VEC>
struct Pack;
template <>
struct Pack<float, 8> {      // 32 bytes in one instruction: two of 16 would touch every sector twice
  float v[8];
  __device__ __forceinline__ void load(const float* p) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                 : "l"(p) : "memory");
  }
  __device__ __forceinline__ void store(float* p) const {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]),
                 "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = v[k];
  }
  __device__ __forceinline__ void set(const float* f) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = f[k];
  }
};
template <>
struct Pack<float, 2> {
  float2 a;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float2*>(p); }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float2*>(p) = a; }
  __device__ __forceinline__ void get(float* f) const { f[0] = a.x; f[1] = a.y; }
  __device__ __forceinline__ void set(const float* f) { a = make_float2(f[0], f[1]); }
};
template <>
struct Pack<float, 1> {
  float a;
  __device__ __forceinline__ void load(const float* p) { a = *p; }
  __device__ __forceinline__ void store(float* p) const { *p = a; }
  __device__ __forceinline__ void get(float* f) const { f[0] = a; }
  __device__ __forceinline__ void set(const float* f) { a = f[0]; }
};
__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {   // ties to even
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
template <>
struct Pack<__nv_bfloat16, 8> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = a; }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = bf16_lo(a.x); f[1] = bf16_hi(a.x); f[2] = bf16_lo(a.y); f[3] = bf16_hi(a.y);
    f[4] = bf16_lo(a.z); f[5] = bf16_hi(a.z); f[6] = bf16_lo(a.w); f[7] = bf16_hi(a.w);
  }
  __device__ __forceinline__ void set(const float* f) {
    a = make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
  }
};
template <>
struct Pack<__nv_bfloat16, 2> {
  uint32_t a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint32_t*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint32_t*>(p) = a; }
  __device__ __forceinline__ void get(float* f) const { f[0] = bf16_lo(a); f[1] = bf16_hi(a); }
  __device__ __forceinline__ void set(const float* f) { a = bf16_pair(f[0], f[1]); }
};
template <>
struct Pack<__nv_bfloat16, 1> {
  __nv_bfloat16 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *p; }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *p = a; }
  __device__ __forceinline__ void get(float* f) const { f[0] = __bfloat162float(a); }
  __device__ __forceinline__ void set(const float* f) { a = __float2bfloat16_rn(f[0]); }
};

// Pairs of fp32, one instruction for both.
__device__ __forceinline__ unsigned long long bits2(float2 a) { return *reinterpret_cast<unsigned long long*>(&a); }
__device__ __forceinline__ float2 pair(unsigned long long u) { return *reinterpret_cast<float2*>(&u); }
__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
  return pair(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
  return pair(r);
}
#endif  // __CUDACC__

}  // namespace lsgd
