// The global norm of many gradient tensors and their clipping.
#include <math.h>

#include <algorithm>

#include "hl_grad.h"
#include "hl_internal.h"
#include "hl_vec.h"

// The tensors of a launch ride in its arguments (no device table to fill, nothing
// that a captured graph or a later call could find changed), as many as 4 KB of
// arguments hold, more in further launches.  Each is cut into chunks, one
// per step of a block, which finds a chunk's tensor by ballots over the tensors' first
// chunks: its lanes hold them.
// Sums take chunks of 16 KB, four loads per thread in flight, a few per block
// (their sums have to be added up); clipping takes 8 KB and a block each.  Over 800
// MB of bf16, chunks of 32, 16 and 8 KB in at most 2048, 4096 and 8192 blocks: sums
// 129, 129 and 126 us, clipping 346, 289 and 270, and 260 with a block per chunk.
template <int MAX, bool DST>
struct gr_args {
  static constexpr int N = MAX;
  static constexpr int CHUNK = DST ? 8192 : 16384;
  static constexpr int PARTS = CHUNK / 16 / 256;  // 16-byte parts of a chunk per thread
  static constexpr uint32_t BLOCKS = DST ? 1u << 20 : 4096;
  const void* src[MAX];
  void* dst[DST ? MAX : 1];
  uint32_t n[MAX];      // elements (GR_PIECE at most), shifted left by two, and the type
  uint32_t c0[MAX];     // first chunk
  int32_t m;            // tensors, or pieces of long ones
  uint32_t chunks;      // in all
};
// (few chunks, up to GR_FEW per block: 600,000 floats 7.0 us, against 3.9 and 1.8 in two launches)
#define GR_FEW 4
#define GR_PIECE (1u << 29)  // (whole chunks)
typedef gr_args<240, false> gr_sq_args;
typedef gr_args<160, true> gr_clip_args;

template <class A>
struct gr_find {
  static constexpr int R = (A::N + 63) / 64;
  uint32_t c[R];  // first chunks of tensors lane, lane + 64, ...
  __device__ __forceinline__ gr_find(const A& g) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int q = 0; q < R; ++q) c[q] = lane + 64 * q < g.m ? g.c0[lane + 64 * q] : ~0u;
  }
  // the last tensor that starts at or before chunk x (an empty one starts where the next does)
  __device__ __forceinline__ int operator()(uint32_t x) const {
    int t = -1;
#pragma unroll
    for (int q = 0; q < R; ++q) t += __popcll(__ballot(c[q] <= x));
    return __builtin_amdgcn_readfirstlane(t);
  }
};

template <class T, class A = gr_sq_args>
__device__ __forceinline__ void gr_sum(const void* src, uint32_t n, uint32_t c, double* acc) {
  constexpr int N = hl_vec<T>::N;
  const T* p = (const T*)src;
  const uint32_t i0 = c * (uint32_t)(A::CHUNK / sizeof(T)) + threadIdx.x * N;
  typename hl_vec<T>::Raw v[A::PARTS];
#pragma unroll
  for (int k = 0; k < A::PARTS; ++k) {
    const uint32_t i = i0 + k * 256 * N;
    v[k] = i < n ? hl_vec<T>::load(p + i, n - i) : hl_vec<T>::zero();
  }
#pragma unroll
  for (int k = 0; k < A::PARTS; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double x = (double)(float)v[k][i];
      acc[i & 3] = fma(x, x, acc[i & 3]);
    }
}

// Squares and sums in 64 bits: an fp32 square overflows from 1.8e19 on.  The
// blocks' sums are added in block order, so the result depends only on the
// tensors' sizes and values: with few blocks by the one that finishes last
// (out), otherwise by gr_total.
__global__ void __launch_bounds__(256)
gr_sq(gr_sq_args g, double* part, uint32_t* ticket, double* out, uint32_t* err) {
  const gr_find<gr_sq_args> find(g);
  double acc[4] = {0., 0., 0., 0.};
  for (uint32_t c = blockIdx.x; c < g.chunks; c += gridDim.x) {
    const int t = find(c);
    const uint32_t n = g.n[t];
    const uint32_t at = c - g.c0[t];
    if ((n & 3) == HL_F32) gr_sum<float>(g.src[t], n >> 2, at, acc);
    else if ((n & 3) == HL_BF16) gr_sum<__bf16>(g.src[t], n >> 2, at, acc);
    else gr_sum<_Float16>(g.src[t], n >> 2, at, acc);
  }
  const double sum = (acc[0] + acc[1]) + (acc[2] + acc[3]);
  double total;
  if (out) {
    if (hl_grid_sum(sum, part, ticket, gridDim.x, err, &total)) *out = total;
    return;
  }
  total = hl_block_sum(sum);
  if (threadIdx.x == 0) part[blockIdx.x] = total;
}

template <class T, class A = gr_clip_args>
__device__ __forceinline__ void gr_scale(const void* src, void* dst, uint32_t n, uint32_t c, hl_clip coef) {
  constexpr int N = hl_vec<T>::N;
  const T* p = (const T*)src;
  T* q = (T*)dst;
  const uint32_t i0 = c * (uint32_t)(A::CHUNK / sizeof(T)) + threadIdx.x * N;
  typename hl_vec<T>::Raw v[A::PARTS];
#pragma unroll
  for (int k = 0; k < A::PARTS; ++k) {
    const uint32_t i = i0 + k * 256 * N;
    if (i < n) v[k] = hl_vec<T>::load(p + i, n - i);
  }
#pragma unroll
  for (int k = 0; k < A::PARTS; ++k) {
    const uint32_t i = i0 + k * 256 * N;
    float o[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      o[j] = coef.f == 0.f ? 0.f : (float)v[k][j] * coef.f;
      if (coef.e) o[j] = ldexpf(o[j], coef.e);
    }
    if (i < n) hl_vec<T>::store(q + i, n - i, hl_vec<T>::pack(o));
  }
}

// The norm's parts and the chunk's tensor are looked up side by side.  The chunks go
// in descending order: gr_sq read them in ascending order, so the memory-side cache
// holds the last ones (107 MB in 701 tensors 57.5 us, in ascending order 60.3).
__global__ void __launch_bounds__(256)
gr_clip(gr_clip_args g, const double* __restrict__ sq, int32_t n_sq, float max_norm, float* norm_out) {
  const gr_find<gr_clip_args> find(g);
  const int t0 = find(g.chunks - 1 - blockIdx.x);
  float norm;
  const hl_clip coef = hl_clip_coef(sq, n_sq, max_norm, &norm);
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
  for (uint32_t i = blockIdx.x; i < g.chunks; i += gridDim.x) {
    const uint32_t c = g.chunks - 1 - i;
    const int t = i == blockIdx.x ? t0 : find(c);
    const uint32_t n = g.n[t];
    const uint32_t at = c - g.c0[t];
    if (coef.f == 1.f && coef.e == 0 && g.src[t] == g.dst[t]) continue;
    if ((n & 3) == HL_F32) gr_scale<float>(g.src[t], g.dst[t], n >> 2, at, coef);
    else if ((n & 3) == HL_BF16) gr_scale<__bf16>(g.src[t], g.dst[t], n >> 2, at, coef);
    else gr_scale<_Float16>(g.src[t], g.dst[t], n >> 2, at, coef);
  }
}

// ----------------------------------------------------------------------------- host side
// The blocks' sums of up to GR_WS_PARTS / BLOCKS launches lie one after another;
// a list of more launches adds them up in between (run).
#define GR_WS_PARTS (8 * gr_sq_args::BLOCKS)
struct gr_ws {
  uint32_t* ticket;
  double *part, *run;
  size_t bytes;
};
static gr_ws gr_carve(void* ws) {
  hl_carver c = hl_carver::after_header(ws, 0);
  gr_ws w;
  w.ticket = c.header() ? c.header() + HL_HDR_GRAD : nullptr;
  w.part = c.take<double>(GR_WS_PARTS);
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

// Fills a launch's arguments with what comes after element *at of tensor *i, and
// moves *i and *at on.
template <class A>
static void gr_fill(A& a, const hl_grad* grads, int32_t n, int32_t* i, int64_t* at) {
  uint32_t c = 0;
  int32_t m = 0;
  for (; m < A::N && *i < n; ++m) {
    const hl_grad& g = grads[*i];
    const size_t es = hl_elem_bytes(g.dtype);
    const uint32_t piece = (uint32_t)std::min<int64_t>(g.n - *at, GR_PIECE);
    a.src[m] = (const char*)g.src + *at * es;
    if (sizeof(a.dst) > sizeof(void*)) a.dst[m] = (char*)g.dst + *at * es;
    a.n[m] = (piece << 2) | (uint32_t)g.dtype;
    a.c0[m] = c;
    c += hl_div_up(piece * (uint64_t)es, A::CHUNK);  // (less than 2^26)
    *at += piece;
    if (*at == g.n) {
      ++*i;
      *at = 0;
    }
  }
  a.m = m;
  a.chunks = c;
}
template <class A>
static uint32_t gr_blocks(const A& a) {
  return std::min(std::max(1u, a.chunks), A::BLOCKS);
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
  gr_sq_args a;
  uint32_t parts = 0;
  bool run = false;
  int32_t i = 0;
  int64_t at = 0;
  for (;;) {
    gr_fill(a, grads, n_grads, &i, &at);
    const bool last = i >= n_grads;
    // a list of few chunks: few blocks, which add their sums up themselves
    const bool alone = last && !parts && !run && a.chunks <= GR_FEW * HL_SUM_TICKETS;
    const uint32_t blocks = alone ? std::min(gr_blocks(a), HL_SUM_TICKETS) : gr_blocks(a);
    HL_KERNEL(h, s, "gr_sq", gr_sq, dim3(blocks), dim3(256), 0, s, a, w.part + parts, w.ticket, alone ? sq : nullptr,
              h->d_err);
    if (alone) break;
    parts += blocks;
    if (last || parts > GR_WS_PARTS - gr_sq_args::BLOCKS) {
      hl_sum_parts(h, w.part, parts, run ? w.run : nullptr, last ? sq : w.run, s);
      parts = 0;
      run = true;
    }
    if (last) break;
  }
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
  gr_clip_args a;
  int32_t i = 0;
  int64_t at = 0;
  do {
    const bool first = i == 0 && at == 0;
    gr_fill(a, grads, n_grads, &i, &at);
    HL_KERNEL(h, s, "gr_clip", gr_clip, dim3(gr_blocks(a)), dim3(256), 0, s, a, sq, n_sq, max_norm,
              first ? norm_out : nullptr);
  } while (i < n_grads);
  HL_LAUNCHED();
  return HL_OK;
}

// ----------------------------------------------------------------------------- parts
__global__ void __launch_bounds__(1024)
gr_total(const double* __restrict__ part, uint32_t n, const double* run, double* out) {
  double x[4] = {0., 0., 0., 0.};
  for (uint32_t i = threadIdx.x; i < n; i += 4096) {
    double y[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] = i + q * 1024 < n ? part[i + q * 1024] : 0.;
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] += y[q];
  }
  const double t = hl_block_sum((x[0] + x[1]) + (x[2] + x[3]));
  if (threadIdx.x == 0) *out = run ? *run + t : t;
}

void hl_sum_parts(const hl_handle* h, const double* part, uint32_t n, const double* run, double* out, hipStream_t s) {
  HL_KERNEL(h, s, "gr_total", gr_total, dim3(1), dim3(1024), 0, s, part, n, run, out);
}
