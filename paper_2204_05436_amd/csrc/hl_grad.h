// Sums over a grid in 64 bits and the clipping coefficient, shared by the dense
// tensors' clipping (hl_grad.hip) and the tables' (hl_embbag.hip).
#pragma once
#include "hl_internal.h"

__device__ __forceinline__ double hl_wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// The sum of v over the block, on thread 0, always in the same order.  Every
// thread of a block of up to 1024 calls it.
__device__ __forceinline__ double hl_block_sum(double v) {
  __shared__ double s_part[16];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = (int)(blockDim.x >> 6);
  v = hl_wave_sum(v);
  if (lane == 0) s_part[w] = v;
  __syncthreads();
  double t = 0.;
  if (threadIdx.x == 0)
    for (int q = 0; q < nw; ++q) t += s_part[q];
  __syncthreads();  // s_part is reused
  return t;
}

// Adds up v over the grid's n blocks in block order: each publishes its sum in
// part[block], and the taker of the last ticket adds them.  True on thread 0 of
// that block, with the sum in *total.  A header that was not zero-filled, or that
// overlapping calls share, hands out tickets past n: HL_DEVERR_INTERNAL.
// The sums are stored and loaded with agent-scope atomics, which bypass the L2s
// that the XCDs do not share, and a block takes its ticket when its store has
// completed: no fence, which would write back and invalidate a whole L2 per block.
// The tickets come one after another, so this is for few blocks (HL_SUM_TICKETS);
// more leave their sums to a launch of their own (hl_sum_parts).  The norm of 213,000
// lookups' gradients, 1,200 blocks: with fences 25.9 us, tickets 19.4, and 5.1 and
// 3.8 with the launch.
#define HL_SUM_TICKETS 64u
void hl_sum_parts(const hl_handle* h, const double* part, uint32_t n, const double* run, double* out, hipStream_t s);
__device__ __forceinline__ bool hl_grid_sum(double v, double* part, uint32_t* ticket, uint32_t n, uint32_t* err,
                                            double* total) {
  __shared__ uint32_t s_last;
  const uint32_t bid = blockIdx.x + gridDim.x * blockIdx.y;
  v = hl_block_sum(v);
  if (n == 1) {
    *total = v;
    return threadIdx.x == 0;
  }
  if (threadIdx.x == 0) {
    __hip_atomic_store(part + bid, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    uint32_t epoch;
    const uint32_t t = hl_ticket(ticket, n, &epoch);
    if (t >= n) hl_flag(err, HL_DEVERR_INTERNAL);
    s_last = t == n - 1;
  }
  __syncthreads();
  if (!s_last) return false;
  double x[4] = {0., 0., 0., 0.};
  for (uint32_t i = threadIdx.x; i < n; i += 4 * blockDim.x) {
    double y[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t j = i + q * blockDim.x;
      y[q] = __hip_atomic_load(part + min(j, n - 1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (j >= n) y[q] = 0.;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] += y[q];
  }
  *total = hl_block_sum((x[0] + x[1]) + (x[2] + x[3]));
  return threadIdx.x == 0;
}

// The norm of a step whose squares add up to sq[0] + ... + sq[n - 1], and the
// factor c that brings it to at most max_norm: 1, or max_norm / norm, or 0 where the
// norm is not finite.  As f * 2^e, e = 0 unless c is so small that fp32 would hold it
// with fewer bits or not at all (the norm may pass 1e38).
// The same on every lane; every lane of a wave calls it.
struct hl_clip {
  float f;
  int e;
};
__device__ __forceinline__ hl_clip hl_clip_coef(const double* sq, int32_t n, float max_norm, float* norm) {
  double s = 0.;
  if (n <= 64) {  // (uniform: few terms, in order)
    for (int32_t i = 0; i < n; ++i) s += sq[i];
  } else {
    for (int32_t i = threadIdx.x & 63; i < n; i += 64) s += sq[i];
    s = hl_wave_sum(s);
  }
  const double d = sqrt(s);
  *norm = (float)d;
  if (!(d <= 1.7976931348623157e308)) return {0.f, 0};
  if (!(d > (double)max_norm)) return {1.f, 0};
  const double c = (double)max_norm / d;
  if (c >= 0x1p-100 || c == 0.) return {(float)c, 0};
  int e;
  const double m = frexp(c, &e);
  return {(float)m, e};
}
