// Rows and tensors of fp32, bf16 or fp16 elements, 16 bytes per lane, shared by
// the routing kernels (hl_route.hip) and the gradient clipping (hl_grad.hip).
#pragma once
#include "hl_internal.h"

#define HL_LINE 128  // bytes of a cache line

// 16 bytes of elements, at any multiple of an element's alignment: the GPU's
// 16-byte loads and stores take any address, so one form serves every row length,
// stride and base.
template <class T>
struct hl_vec {
  static constexpr int N = 16 / (int)sizeof(T);
  typedef T Raw __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
  static __device__ __forceinline__ Raw zero() {
    Raw r;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = (T)0.f;
    return r;
  }
  // Elements [0, n) of p (the others zero); n >= N: all of them.
  // HINT (non-temporal): for what a launch reads or writes once, so that it does not
  // displace other lines in the L2s: rows' sums of 537 MB 127 us without it, 115 with
  // it on loads and stores.
  template <bool HINT = true>
  static __device__ __forceinline__ Raw load(const T* p, int64_t n) {
    if (n >= N) {
      const Raw* q = reinterpret_cast<const Raw*>(p);
      return HINT ? __builtin_nontemporal_load(q) : *q;
    }
    Raw r = zero();
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (i < n) r[i] = p[i];
    return r;
  }
  template <bool HINT = true>
  static __device__ __forceinline__ void store(T* p, int64_t n, const Raw& r) {
    if (n >= N) {
      if (HINT) __builtin_nontemporal_store(r, reinterpret_cast<Raw*>(p));
      else *reinterpret_cast<Raw*>(p) = r;
      return;
    }
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (i < n) p[i] = r[i];
  }
  // rounded to nearest even by the hardware's conversion (NaN stays NaN)
  static __device__ __forceinline__ Raw pack(const float* v) {
    Raw r;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = (T)v[i];
    return r;
  }
};

static inline size_t hl_elem_bytes(int32_t dtype) {
  return dtype == HL_F32 ? 4 : (dtype == HL_BF16 || dtype == HL_F16 ? 2 : 0);
}

// F<T>(args) for the element type that dtype names
#define HL_BY_TYPE(dtype, F, ...)                        \
  do {                                                   \
    if ((dtype) == HL_F32) F<float>(__VA_ARGS__);        \
    else if ((dtype) == HL_BF16) F<__bf16>(__VA_ARGS__); \
    else F<_Float16>(__VA_ARGS__);                       \
  } while (0)
