// The global norm of many gradient tensors and their clipping.
#include <math.h>

#include <algorithm>

#include "hl_grad.h"
#include "hl_internal.h"
#include "hl_vec.h"

// The tensors of a launch ride in its arguments (no device table to fill, nothing
// that a captured graph or a later call could find changed): GR_MAX of them, more
// in further launches.  Each is cut into chunks of GR_CHUNK bytes, one per step of
// a block; a block takes consecutive chunks, and finds the tensor of each by two
// ballots over the tensors' first chunks, which its lanes hold.
#define GR_MAX 112
#define GR_CHUNK 32768
#define GR_PARTS (GR_CHUNK / 16 / 256)  // 16-byte parts of a chunk per thread
#define GR_BLOCKS 2048

struct gr_ent {
  const void* src;
  void* dst;
  int64_t n;
  uint32_t c0;  // first chunk
  int32_t dtype;
};
struct gr_args {
  gr_ent e[GR_MAX];
};

struct gr_find {
  uint32_t a, b;  // first chunks of tensors lane and lane + 64
  __device__ __forceinline__ gr_find(const gr_args& g, int m) {
    const int lane = threadIdx.x & 63;
    a = lane < m ? g.e[lane].c0 : ~0u;
    b = lane + 64 < m ? g.e[lane + 64].c0 : ~0u;
  }
  // the last tensor that starts at or before chunk c (an empty one starts where the next does)
  __device__ __forceinline__ int operator()(uint32_t c) const {
    return __popcll(__ballot(a <= c)) + __popcll(__ballot(b <= c)) - 1;
  }
};

template <class T>
__device__ __forceinline__ void gr_sum(const gr_ent& e, uint32_t c, double* acc) {
  constexpr int N = hl_vec<T>::N;
  const T* p = (const T*)e.src;
  const int64_t i0 = (int64_t)(c - e.c0) * (GR_CHUNK / sizeof(T)) + threadIdx.x * N;
  typename hl_vec<T>::Raw v[GR_PARTS];
#pragma unroll
  for (int k = 0; k < GR_PARTS; ++k) {
    const int64_t i = i0 + (int64_t)k * 256 * N;
    v[k] = i < e.n ? hl_vec<T>::load(p + i, e.n - i) : hl_vec<T>::zero();
  }
#pragma unroll
  for (int k = 0; k < GR_PARTS; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double x = (double)(float)v[k][i];
      acc[i & 3] = fma(x, x, acc[i & 3]);
    }
}

// Squares and sums in 64 bits: an fp32 square overflows from 1.8e19 on.  The
// blocks' sums are added in block order by the block that finishes last, so the
// result depends only on the tensors' sizes and values.
__global__ void __launch_bounds__(256)
gr_sq(gr_args g, int m, uint32_t chunks, uint32_t per, double* part, uint32_t* ticket, double* run, int first,
      double* out, uint32_t* err) {
  const gr_find find(g, m);
  double acc[4] = {0., 0., 0., 0.};
  const uint32_t c1 = min(chunks, (blockIdx.x + 1) * per);
  for (uint32_t c = blockIdx.x * per; c < c1; ++c) {
    const gr_ent& e = g.e[__builtin_amdgcn_readfirstlane(find(c))];
    if (e.dtype == HL_F32) gr_sum<float>(e, c, acc);
    else if (e.dtype == HL_BF16) gr_sum<__bf16>(e, c, acc);
    else gr_sum<_Float16>(e, c, acc);
  }
  double total;
  if (hl_grid_sum((acc[0] + acc[1]) + (acc[2] + acc[3]), part, ticket, gridDim.x, err, &total)) {
    if (!first) total += *run;
    if (out) *out = total;
    else *run = total;
  }
}

template <class T>
__device__ __forceinline__ void gr_scale(const gr_ent& e, uint32_t c, float coef) {
  constexpr int N = hl_vec<T>::N;
  const T* p = (const T*)e.src;
  T* q = (T*)e.dst;
  const int64_t i0 = (int64_t)(c - e.c0) * (GR_CHUNK / sizeof(T)) + threadIdx.x * N;
  typename hl_vec<T>::Raw v[GR_PARTS];
#pragma unroll
  for (int k = 0; k < GR_PARTS; ++k) {
    const int64_t i = i0 + (int64_t)k * 256 * N;
    if (i < e.n) v[k] = hl_vec<T>::load(p + i, e.n - i);
  }
#pragma unroll
  for (int k = 0; k < GR_PARTS; ++k) {
    const int64_t i = i0 + (int64_t)k * 256 * N;
    float o[N];
#pragma unroll
    for (int j = 0; j < N; ++j) o[j] = coef == 0.f ? 0.f : (float)v[k][j] * coef;
    if (i < e.n) hl_vec<T>::store(q + i, e.n - i, hl_vec<T>::pack(o));
  }
}

__global__ void __launch_bounds__(256)
gr_clip(gr_args g, int m, uint32_t chunks, uint32_t per, const double* __restrict__ sq, int32_t n_sq, float max_norm,
        float* norm_out) {
  float norm;
  const float coef = hl_clip_coef(sq, n_sq, max_norm, &norm);
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
  const gr_find find(g, m);
  const uint32_t c1 = min(chunks, (blockIdx.x + 1) * per);
  for (uint32_t c = blockIdx.x * per; c < c1; ++c) {
    const gr_ent& e = g.e[__builtin_amdgcn_readfirstlane(find(c))];
    if (coef == 1.f && e.src == e.dst) continue;
    if (e.dtype == HL_F32) gr_scale<float>(e, c, coef);
    else if (e.dtype == HL_BF16) gr_scale<__bf16>(e, c, coef);
    else gr_scale<_Float16>(e, c, coef);
  }
}

// ----------------------------------------------------------------------------- host side
struct gr_ws {
  uint32_t* ticket;
  double *part, *run;
  size_t bytes;
};
static gr_ws gr_carve(void* ws) {
  hl_carver c = hl_carver::after_header(ws, 0);
  gr_ws w;
  w.ticket = c.header() ? c.header() + HL_HDR_GRAD : nullptr;
  w.part = c.take<double>(GR_BLOCKS);
  w.run = c.take<double>(1);
  w.bytes = c.off;
  return w;
}

extern "C" size_t hl_grad_workspace_bytes(void) { return (gr_carve(nullptr).bytes + 255) & ~(size_t)255; }

// HL_OK if every tensor is one that the calls take
static hl_status gr_check(const hl_handle* h, const hl_grad* grads, int32_t n, bool write) {
  if (!h || n < 0 || (n > 0 && !grads)) return HL_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n; ++i) {
    const hl_grad& g = grads[i];
    const size_t es = hl_elem_bytes(g.dtype);
    if (!es || g.n < 0) return HL_ERR_INVALID_ARG;
    if (g.n > (1ll << 40)) return HL_ERR_UNSUPPORTED;
    if (g.n == 0) continue;
    if (!g.src || (uintptr_t)g.src % es != 0) return HL_ERR_INVALID_ARG;
    if (write) {
      if (!g.dst || (uintptr_t)g.dst % es != 0) return HL_ERR_INVALID_ARG;
      const uintptr_t a = (uintptr_t)g.src, b = (uintptr_t)g.dst, len = (uintptr_t)g.n * es;
      if (a != b && a < b + len && b < a + len) return HL_ERR_INVALID_ARG;  // they overlap in part
    }
  }
  return hl_on_device(h);
}

// Fills a launch's arguments with the tensors from grads[i] on; returns their number.
static int32_t gr_fill(gr_args& a, const hl_grad* grads, int32_t i, int32_t n, uint32_t* chunks) {
  uint32_t c = 0;
  int32_t m = 0;
  for (; m < GR_MAX && i + m < n; ++m) {
    const hl_grad& g = grads[i + m];
    const uint64_t need = ((uint64_t)g.n * hl_elem_bytes(g.dtype) + GR_CHUNK - 1) / GR_CHUNK;
    if (m > 0 && c + need > 0x7FFFFFFFull) break;  // (a tensor alone has fewer than 2^28)
    a.e[m] = {g.src, g.dst, g.n, c, g.dtype};
    c += (uint32_t)need;
  }
  *chunks = c;
  return m;
}

extern "C" hl_status hl_grad_sq(hl_handle* h, const hl_grad* grads, int32_t n_grads, double* sq, void* workspace,
                                size_t ws_bytes, hl_stream stream) {
  hl_status st = gr_check(h, grads, n_grads, false);
  if (st != HL_OK) return st;
  if (!sq || (uintptr_t)sq % 8 != 0 || !workspace || (uintptr_t)workspace % 8 != 0) return HL_ERR_INVALID_ARG;
  if (ws_bytes < hl_grad_workspace_bytes()) return HL_ERR_CAPACITY;
  hl_ws_note(h, workspace, HL_WSK_OTHER);
  const gr_ws w = gr_carve(workspace);
  hipStream_t s = (hipStream_t)stream;
  gr_args a;
  int32_t i = 0;
  do {
    uint32_t chunks = 0;
    const int32_t m = gr_fill(a, grads, i, n_grads, &chunks);
    const uint32_t per = std::max(1u, hl_div_up(chunks, GR_BLOCKS));
    const uint32_t blocks = std::max(1u, hl_div_up(chunks, per));
    HL_KERNEL(h, s, "gr_sq", gr_sq, dim3(blocks), dim3(256), 0, s, a, m, chunks, per, w.part, w.ticket, w.run,
              (int)(i == 0), i + m >= n_grads ? sq : nullptr, h->d_err);
    i += m;
  } while (i < n_grads);
  HL_LAUNCHED();
  return HL_OK;
}

extern "C" hl_status hl_grad_clip(const hl_handle* h, const hl_grad* grads, int32_t n_grads, const double* sq,
                                  int32_t n_sq, float max_norm, float* norm_out, hl_stream stream) {
  hl_status st = gr_check(h, grads, n_grads, true);
  if (st != HL_OK) return st;
  if (!sq || (uintptr_t)sq % 8 != 0 || n_sq < 1 || !(max_norm >= 0.f) || (uintptr_t)norm_out % 4 != 0)
    return HL_ERR_INVALID_ARG;
  hipStream_t s = (hipStream_t)stream;
  gr_args a;
  int32_t i = 0;
  do {
    uint32_t chunks = 0;
    const int32_t m = gr_fill(a, grads, i, n_grads, &chunks);
    const uint32_t per = std::max(1u, hl_div_up(chunks, GR_BLOCKS));
    const uint32_t blocks = std::max(1u, hl_div_up(chunks, per));
    HL_KERNEL(h, s, "gr_clip", gr_clip, dim3(blocks), dim3(256), 0, s, a, m, chunks, per, sq, n_sq, max_norm,
              i == 0 ? norm_out : nullptr);
    i += m;
  } while (i < n_grads);
  HL_LAUNCHED();
  return HL_OK;
}
