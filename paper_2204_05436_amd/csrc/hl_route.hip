// Rows sent to experts and back: a stable counting sort of the assignments by
// expert (hl_route_plan), and the row movements it directs, each with its
// gradient.
#include <algorithm>

#include "hl_internal.h"
#include "hl_vec.h"

// ----------------------------------------------------------------------------- plan
// Stable counting sort of N = n_tokens * k expert ids.  A block takes a tile of
// RT_THREADS * ITEMS consecutive assignments, each of its waves a consecutive
// part, 64 at a time: the lanes that name the same expert find each other by
// ballots, the running count of the wave's part gives an assignment its rank
// there, and the counts of the waves before, of the tiles before and of the
// experts before (capped and rounded up) give the row.  Up to RT_ONE assignments
// are one tile and one launch.  More take a launch that counts the tiles first;
// every tile then adds up the counts it needs, or past RT_DIRECT counts a third
// launch turns them into prefixes.  Bound by latency: the launches, and in each the
// ids, the ballots, three barriers and the scattered rows.
// In a graph, us per plan: 1 tile of 4096 ids of 8, 64, 256 and 1024 experts 5.8, 6.5,
// 7.4 and 9.0, of 8192 8.5, 9.9, 11.6 and 13.7 where two launches take 6.4, 6.6, 7.8
// and 11.8.  65,536 ids: 6.7, 8.0, 10.2, 13.2 (64 tiles of 1024 experts without the
// third launch 27.7; of 64 with it 9.2).  1,048,576 ids: 11.6, 16.8, 19.9, 29.4 in
// 256 tiles, 15.1, 20.9, 24.9, 30.6 in 128.
#define RT_THREADS 1024
#define RT_WAVES (RT_THREADS / 64)
#define RT_MAX_EXPERTS 1024
#define RT_MAX_DIM (1 << 20)
#define RT_ONE 4096
#define RT_TILES 256
#define RT_DIRECT 8192

struct rt_shape {
  int32_t n;       // assignments
  int32_t E, bits; // experts; bits of an expert id
  int32_t cap;     // INT32_MAX: none
  int32_t align;
  int64_t rows;    // rows of the caller's buffers
};

// The assignments of one tile: valid expert ids in ex (else -1), each one's rank
// among those of its wave's part in rk, and the parts' counts in cnt[wave][E].
template <int ITEMS>
__device__ __forceinline__ void rt_count(const int32_t* __restrict__ experts, const rt_shape& sh, uint32_t tile,
                                         volatile uint16_t* cnt, int32_t* ex, uint32_t* rk, uint32_t* err) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t i0 = (int64_t)tile * (RT_THREADS * ITEMS) + w * (64 * ITEMS) + lane;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int64_t a = i0 + i * 64;
    ex[i] = a < sh.n ? experts[a] : -1;
  }
  volatile uint16_t* mine = cnt + w * sh.E;
  for (int e = lane; e < sh.E; e += 64) mine[e] = 0;
  const uint64_t below = (1ull << lane) - 1ull;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const bool in = (uint32_t)ex[i] < (uint32_t)sh.E;
    if (!in && ex[i] != -1) hl_flag(err, HL_DEVERR_OUT_OF_RANGE);
    if (!in) ex[i] = -1;
    const uint64_t m = hl_match_digit((uint32_t)ex[i], sh.bits, in);
    uint32_t before = 0;
    if (in) before = mine[ex[i]];
    rk[i] = before + (uint32_t)__popcll(m & below);
    __builtin_amdgcn_wave_barrier();  // (every lane has read the count before its first lane of the expert raises it)
    if (in && (m & below) == 0) mine[ex[i]] = (uint16_t)(before + (uint32_t)__popcll(m));
    __builtin_amdgcn_wave_barrier();
  }
}

template <int ITEMS>
__global__ void __launch_bounds__(RT_THREADS)
rt_tiles(const int32_t* __restrict__ experts, rt_shape sh, uint32_t* __restrict__ hist, uint32_t* err) {
  extern __shared__ uint16_t s_cnt[];
  int32_t ex[ITEMS];
  uint32_t rk[ITEMS];
  rt_count<ITEMS>(experts, sh, blockIdx.x, s_cnt, ex, rk, err);
  __syncthreads();
  for (int e = threadIdx.x; e < sh.E; e += RT_THREADS) {
    uint32_t t = 0;
#pragma unroll
    for (int w = 0; w < RT_WAVES; ++w) t += s_cnt[w * sh.E + e];
    hist[(size_t)blockIdx.x * sh.E + e] = t;
  }
}

// hist[tile][e] becomes the count of expert e in the tiles before; hist[tiles][e]
// the count in all of them.  A block per expert.
__global__ void __launch_bounds__(256)
rt_prefix(uint32_t* hist, uint32_t tiles, int32_t E) {
  __shared__ uint32_t s_w[4];
  const int e = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t run = 0;
  for (uint32_t t0 = 0; t0 < tiles; t0 += 256) {
    const uint32_t t = t0 + threadIdx.x;
    const uint32_t c = t < tiles ? hist[(size_t)t * E + e] : 0u;
    uint32_t x = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    if (lane == 63) s_w[w] = x;
    __syncthreads();
    uint32_t before = run, all = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q < w) before += s_w[q];
      all += s_w[q];
    }
    if (t < tiles) hist[(size_t)t * E + e] = before + x - c;
    run += all;
    __syncthreads();  // s_w is reused
  }
  if (threadIdx.x == 0) hist[(size_t)tiles * E + e] = run;
}

// hist: the tiles' counts (mode 1) or prefixes with the totals (mode 2), unused
// for a single tile (mode 0).
template <int ITEMS>
__global__ void __launch_bounds__(RT_THREADS)
rt_place(const int32_t* __restrict__ experts, rt_shape sh, const uint32_t* __restrict__ hist, uint32_t tiles, int mode,
         int32_t* __restrict__ counts, int32_t* __restrict__ offsets, int32_t* __restrict__ pos,
         int32_t* __restrict__ order, uint32_t* err) {
  extern __shared__ uint32_t s_dyn[];
  uint32_t *s_prev = s_dyn, *s_tot = s_prev + sh.E, *s_off = s_tot + sh.E;  // [E], [E], [E + 1]
  uint16_t* s_cnt = reinterpret_cast<uint16_t*>(s_off + sh.E + 1);           // [RT_WAVES][E]
  __shared__ uint32_t s_w[RT_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const uint32_t tile = blockIdx.x;
  if (tid < sh.E) s_prev[tid] = s_tot[tid] = 0;
  // the tiles' counts, loaded beside the ids: every thread adds up some tiles of one expert
  uint32_t prev = 0, tot = 0;
  const int he = tid & ((1 << sh.bits) - 1);
  if (mode == 1 && he < sh.E) {
    const uint32_t segs = RT_THREADS >> sh.bits;
#pragma unroll 8
    for (uint32_t t = (uint32_t)tid >> sh.bits; t < tiles; t += segs) {
      const uint32_t c = hist[(size_t)t * sh.E + he];
      tot += c;
      if (t < tile) prev += c;
    }
  }
  int32_t ex[ITEMS];
  uint32_t rk[ITEMS];
  rt_count<ITEMS>(experts, sh, tile, s_cnt, ex, rk, err);
  __syncthreads();
  // the parts' counts become those of the parts before
  uint32_t mine = 0;
  if (tid < sh.E) {
#pragma unroll
    for (int q = 0; q < RT_WAVES; ++q) {
      const uint32_t c = s_cnt[q * sh.E + tid];
      s_cnt[q * sh.E + tid] = (uint16_t)mine;
      mine += c;
    }
  }
  if (mode == 1) {
    if (tot) atomicAdd(&s_tot[he], tot);
    if (prev) atomicAdd(&s_prev[he], prev);
  } else if (tid < sh.E) {
    s_prev[tid] = mode == 2 ? hist[(size_t)tile * sh.E + tid] : 0u;
    s_tot[tid] = mode == 2 ? hist[(size_t)tiles * sh.E + tid] : mine;
  }
  __syncthreads();
  // the experts' blocks, one after another
  uint32_t kept = 0, block = 0;
  if (tid < sh.E) {
    kept = min(s_tot[tid], (uint32_t)sh.cap);
    block = (kept + sh.align - 1) / sh.align * sh.align;
  }
  uint32_t x = block;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  if (lane == 63) s_w[w] = x;
  __syncthreads();
  for (int q = 0; q < w; ++q) x += s_w[q];
  if (tid < sh.E) {
    s_off[tid] = x - block;
    if (tid == sh.E - 1) s_off[sh.E] = x;
    if (tile == 0) {
      counts[tid] = (int32_t)kept;
      offsets[tid] = (int32_t)(x - block);
      if (tid == sh.E - 1) offsets[sh.E] = (int32_t)x;
    }
  }
  __syncthreads();
  const int64_t i0 = (int64_t)tile * (RT_THREADS * ITEMS) + w * (64 * ITEMS) + lane;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int64_t a = i0 + i * 64;
    int32_t p = -1;
    if (ex[i] >= 0) {
      const uint32_t rank = s_prev[ex[i]] + s_cnt[w * sh.E + ex[i]] + rk[i];
      if (rank < (uint32_t)sh.cap) {
        p = (int32_t)(s_off[ex[i]] + rank);
        if ((int64_t)p >= sh.rows) {  // (hl_route_rows bounds it)
          hl_flag(err, HL_DEVERR_INTERNAL);
          p = -1;
        }
      }
    }
    if (a < sh.n) pos[a] = p;
    if (p >= 0 && order) order[p] = (int32_t)a;
  }
  if (order && sh.align > 1)
    for (uint32_t e = tile; e < (uint32_t)sh.E; e += tiles) {
      const uint32_t end = min((int64_t)s_off[e + 1], sh.rows);
      for (uint32_t r = s_off[e] + min(s_tot[e], (uint32_t)sh.cap) + tid; r < end; r += RT_THREADS) order[r] = -1;
    }
}

// assignments per thread: as few as keep the tiles to one, else to RT_TILES
static int rt_items(int64_t n) {
  int items = 1;
  while (items < 8 && n > (n <= RT_ONE ? 1 : RT_TILES) * (int64_t)RT_THREADS * items) items *= 2;
  return items;
}
static uint32_t rt_tile_count(int64_t n) {
  return n ? hl_div_up((uint64_t)n, (uint64_t)RT_THREADS * rt_items(n)) : 1;
}

// ----------------------------------------------------------------------------- row movements
// All of these are bound by memory: a row's 16-byte parts lie one per lane.  2^lg
// lanes take a token's chunk of that many parts, so a block of 256 holds several
// short rows or 256 parts (4 KB) of one, whose further chunks are the next blocks'.
// Neighbouring blocks thus read and write the same rows at the same time; a wave per
// KB of a row with the rows' pieces far apart in time took 155 us instead of 127 for
// the sums of 4 rows of 8 KB of 16,384 tokens.
// UNI: a wave's lanes all hold the same token (lg >= 6), whose rows' addresses are
// then scalar.  KB: assignments of a token whose rows are in flight together.  HINT:
// the non-temporal hint on the experts' rows, where those are whole cache lines
// (neighbouring rows that share lines are better left to the L2s).  In TB/s of what
// has to be read and written, gather, combine and combine_bwd: 16,384 tokens of 8 KB
// in bf16 to 4 experts 5.6, 5.7, 5.9 (without the hint 5.5, 5.5, 5.2); 30,000 of 1 KB
// to 2 6.0, 5.1, 5.6 (4.8, 5.2, 5.4); 2,999 of 3,076 bytes to 6, which share lines,
// 4.7, 4.2, 4.1 (with it 3.9, 4.1, 3.7).  A copy of 537 MB reaches 5.4 here.
struct rt_geom {
  int32_t dim, k, lg, chunks;  // lg: log2 of the lanes of a chunk; chunks per row
  int64_t n_tokens, rows;
  int32_t n_experts;
};

// Blocks in x and y together: a grid's x may not hold more than 2^32 threads.
__device__ __forceinline__ uint32_t rt_block() { return blockIdx.x + blockIdx.y * gridDim.x; }
// This lane's token and column; false: none.
template <class T, bool UNI>
__device__ __forceinline__ bool rt_part(const rt_geom& g, uint32_t* t, int32_t* col) {
  uint32_t u, l;
  if (UNI) {
    const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    u = rt_block() * (256u >> g.lg) + (w >> (g.lg - 6));
    l = ((w & ((1u << (g.lg - 6)) - 1)) << 6) + (threadIdx.x & 63);
  } else {
    u = rt_block() * (256u >> g.lg) + (threadIdx.x >> g.lg);
    l = threadIdx.x & ((1u << g.lg) - 1);
  }
  uint32_t c = 0;
  *t = u;
  if (g.chunks > 1) {
    *t = u / (uint32_t)g.chunks;
    c = u - *t * (uint32_t)g.chunks;
  }
  *col = (int32_t)(((c << g.lg) + l) * hl_vec<T>::N);
  return *t < g.n_tokens && *col < g.dim;
}
template <bool UNI>
__device__ __forceinline__ int32_t rt_row(int32_t p, int64_t rows, uint32_t* err) {
  if (UNI) p = __builtin_amdgcn_readfirstlane(p);
  if (p == -1) return -1;
  if (p < 0 || p >= rows) {
    hl_flag(err, HL_DEVERR_BAD_CODE);
    return -1;
  }
  return p;
}
// The padding rows of expert e's block, set to zero.
template <class T>
__device__ __forceinline__ void rt_pad(uint32_t e, const int32_t* __restrict__ counts,
                                       const int32_t* __restrict__ offsets, const rt_geom& g, T* __restrict__ out,
                                       int64_t stride) {
  constexpr int N = hl_vec<T>::N;
  if (e >= (uint32_t)g.n_experts) return;
  const int64_t end = min((int64_t)offsets[e + 1], g.rows);
  for (int64_t r = max((int64_t)offsets[e] + counts[e], (int64_t)0) + (threadIdx.x >> g.lg); r < end; r += 256 >> g.lg)
    for (int64_t col = (int64_t)(threadIdx.x & ((1 << g.lg) - 1)) * N; col < g.dim; col += (int64_t)N << g.lg)
      hl_vec<T>::store(out + r * stride + col, g.dim - col, hl_vec<T>::zero());
}

// A token's row is loaded once and stored k times.
template <class T, bool UNI, int KB, bool HINT>
__global__ void __launch_bounds__(256)
rt_gather(rt_geom g, uint32_t blocks, const int32_t* __restrict__ pos, const int32_t* __restrict__ counts,
          const int32_t* __restrict__ offsets, const T* __restrict__ x, int64_t xs, T* __restrict__ out, int64_t os,
          uint32_t* err) {
  if (rt_block() >= blocks) {
    rt_pad<T>(rt_block() - blocks, counts, offsets, g, out, os);
    return;
  }
  uint32_t t;
  int32_t col;
  if (!rt_part<T, UNI>(g, &t, &col)) return;
  const int64_t n = g.dim - col;
  const typename hl_vec<T>::Raw v = hl_vec<T>::template load<false>(x + t * xs + col, n);
  const int32_t* pt = pos + (int64_t)t * g.k;
  for (int j0 = 0; j0 < g.k; j0 += KB) {
    int32_t p[KB];
#pragma unroll
    for (int j = 0; j < KB; ++j) p[j] = j0 + j < g.k ? pt[j0 + j] : -1;
#pragma unroll
    for (int j = 0; j < KB; ++j) {
      p[j] = rt_row<UNI>(p[j], g.rows, err);
      if (p[j] >= 0) hl_vec<T>::template store<HINT>(out + (int64_t)p[j] * os + col, n, v);
    }
  }
}

template <class T, bool UNI, int KB, bool W, bool HINT>
__global__ void __launch_bounds__(256)
rt_combine(rt_geom g, const int32_t* __restrict__ pos, const T* __restrict__ rows, int64_t rs,
           const float* __restrict__ weights, T* __restrict__ out, int64_t os, uint32_t* err) {
  typedef typename hl_vec<T>::Raw Raw;
  constexpr int N = hl_vec<T>::N;
  uint32_t t;
  int32_t col;
  if (!rt_part<T, UNI>(g, &t, &col)) return;
  const int64_t n = g.dim - col;
  const int32_t* pt = pos + (int64_t)t * g.k;
  const float* wt = W ? weights + (int64_t)t * g.k : nullptr;
  float acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = 0.f;
  for (int j0 = 0; j0 < g.k; j0 += KB) {
    int32_t p[KB];
    float w[KB];
    Raw v[KB];
#pragma unroll
    for (int j = 0; j < KB; ++j) {
      p[j] = j0 + j < g.k ? pt[j0 + j] : -1;
      w[j] = W && j0 + j < g.k ? wt[j0 + j] : 1.f;
    }
#pragma unroll
    for (int j = 0; j < KB; ++j) {
      p[j] = rt_row<UNI>(p[j], g.rows, err);
      if (p[j] >= 0) v[j] = hl_vec<T>::template load<HINT>(rows + (int64_t)p[j] * rs + col, n);
    }
#pragma unroll
    for (int j = 0; j < KB; ++j)
      if (p[j] >= 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = W ? fmaf(w[j], (float)v[j][i], acc[i]) : acc[i] + (float)v[j][i];
      }
  }
  hl_vec<T>::store(out + t * os + col, n, hl_vec<T>::pack(acc));
}

// The gradients of the weighted sum: an assignment's row of drows is w times the
// token's gradient, its weight's gradient their dot product.  The lanes of a
// chunk take all of the token's chunks in turn, and add their dot products up at
// the end.  (No hint on dout: with it 58.9 us instead of 51.5 for 8,192 tokens of 8 KB
// to 2 experts.)
template <class T, bool UNI, int KB, bool HINT>
__global__ void __launch_bounds__(256)
rt_combine_bwd(rt_geom g, uint32_t blocks, const int32_t* __restrict__ pos, const int32_t* __restrict__ counts,
               const int32_t* __restrict__ offsets, const T* __restrict__ dout, int64_t ds,
               const T* __restrict__ rows, int64_t rs, const float* __restrict__ weights, T* __restrict__ drows,
               int64_t drs, float* __restrict__ dweights, uint32_t* err) {
  typedef typename hl_vec<T>::Raw Raw;
  constexpr int N = hl_vec<T>::N;
  __shared__ float s_dot[4][KB];
  if (rt_block() >= blocks) {
    rt_pad<T>(rt_block() - blocks, counts, offsets, g, drows, drs);
    return;
  }
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t t;
  int32_t c0;
  rt_geom g1 = g;
  g1.chunks = 1;
  rt_part<T, UNI>(g1, &t, &c0);
  const bool in = t < g.n_tokens;
  const int32_t* pt = pos + (int64_t)t * g.k;
  for (int j0 = 0; j0 < g.k; j0 += KB) {
    int32_t p[KB];
    float wt[KB], dot[KB];
#pragma unroll
    for (int j = 0; j < KB; ++j) {
      const bool has = in && j0 + j < g.k;
      p[j] = has ? pt[j0 + j] : -1;
      wt[j] = has && weights ? weights[(int64_t)t * g.k + j0 + j] : 1.f;
      dot[j] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < KB; ++j) p[j] = rt_row<UNI>(p[j], g.rows, err);
    if (in)
      for (int32_t col = c0; col < g.dim; col += N << g.lg) {
        const int64_t n = g.dim - col;
        const Raw d = hl_vec<T>::template load<false>(dout + t * ds + col, n);
        Raw v[KB];
        if (dweights)
#pragma unroll
          for (int j = 0; j < KB; ++j)
            if (p[j] >= 0) v[j] = hl_vec<T>::template load<HINT>(rows + (int64_t)p[j] * rs + col, n);
#pragma unroll
        for (int j = 0; j < KB; ++j)
          if (p[j] >= 0) {
            float o[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
              o[i] = wt[j] * (float)d[i];
              if (dweights) dot[j] = fmaf((float)d[i], (float)v[j][i], dot[j]);
            }
            hl_vec<T>::store(drows + (int64_t)p[j] * drs + col, n, hl_vec<T>::pack(o));
          }
      }
    if (!dweights) continue;
    const int lg = UNI ? 6 : g.lg;
    for (int o = 1; o < (1 << lg); o <<= 1)
#pragma unroll
      for (int j = 0; j < KB; ++j) dot[j] += __shfl_xor(dot[j], o);
    if (UNI && g.lg > 6) {  // a token's waves, in order
      if (lane == 0)
#pragma unroll
        for (int j = 0; j < KB; ++j) s_dot[w][j] = dot[j];
      __syncthreads();
      const int wpt = 1 << (g.lg - 6);
      if (in && (w & (wpt - 1)) == 0 && lane < KB && j0 + lane < g.k) {
        float s = 0.f;
        for (int q = 0; q < wpt; ++q) s += s_dot[w + q][lane];
        dweights[(int64_t)t * g.k + j0 + lane] = s;
      }
      __syncthreads();
    } else if (in && (lane & ((1 << lg) - 1)) == 0) {
#pragma unroll
      for (int j = 0; j < KB; ++j)
        if (j0 + j < g.k) dweights[(int64_t)t * g.k + j0 + j] = dot[j];
    }
  }
}

// ----------------------------------------------------------------------------- host side
extern "C" int64_t hl_route_rows(int64_t n_tokens, int32_t k, int32_t n_experts, int32_t capacity, int32_t align) {
  if (n_tokens < 0 || k < 1 || n_experts < 1 || capacity < 0 || align < 1) return 0;
  if (n_tokens > (1ll << 30) || n_tokens * k > (1ll << 30)) return 0;
  const int64_t n = n_tokens * k, most = capacity ? std::min<int64_t>(capacity, n) : n;
  return std::min(n + std::min<int64_t>(n_experts, n) * (align - 1), n_experts * ((most + align - 1) / align * align));
}

extern "C" size_t hl_route_workspace_bytes(int64_t n_tokens, int32_t k, int32_t n_experts) {
  if (n_tokens < 0 || k < 1 || n_experts < 1 || n_experts > RT_MAX_EXPERTS) return 0;
  if (n_tokens > (1ll << 30) || n_tokens * k > (1ll << 30)) return 0;
  hl_carver c = hl_carver::after_header(nullptr, 0);
  c.take<uint32_t>(((size_t)rt_tile_count(n_tokens * k) + 1) * n_experts);
  return (c.off + 255) & ~(size_t)255;
}

static hl_status rt_check(const hl_handle* h, const hl_route* r) {
  if (!h || !r) return HL_ERR_INVALID_ARG;
  if (r->n_tokens < 0 || r->k < 1 || r->n_experts < 1 || r->capacity < 0 || r->align < 1) return HL_ERR_INVALID_ARG;
  if (!r->counts || !r->offsets || (r->n_tokens > 0 && !r->pos)) return HL_ERR_INVALID_ARG;
  if (r->n_tokens > (1ll << 30) || r->n_tokens * r->k > (1ll << 30) || r->n_experts > RT_MAX_EXPERTS)
    return HL_ERR_UNSUPPORTED;
  const int64_t need = hl_route_rows(r->n_tokens, r->k, r->n_experts, r->capacity, r->align);
  if (need >= (1ll << 31)) return HL_ERR_UNSUPPORTED;
  if (r->n_rows < need) return HL_ERR_CAPACITY;
  return hl_on_device(h);
}
// a row buffer: its pointer, and a stride of at least a row
static hl_status rt_rows_ok(const void* p, int64_t stride, int32_t dim, size_t es) {
  if (!p || (uintptr_t)p % es != 0 || stride < dim || stride > (1ll << 31)) return HL_ERR_INVALID_ARG;
  return HL_OK;
}
static hl_status rt_check_rows(const hl_handle* h, const hl_route* r, int32_t dtype, int32_t dim, const void* a,
                               int64_t as, const void* b, int64_t bs) {
  hl_status st = rt_check(h, r);
  if (st != HL_OK) return st;
  const size_t es = hl_elem_bytes(dtype);
  if (!es || dim < 1) return HL_ERR_INVALID_ARG;
  // (blocks of 4 KB of a row: fewer than 2^31, 8 TB of tokens)
  if (dim > RT_MAX_DIM || r->n_tokens * (int64_t)hl_div_up(dim * es, 4096) >= (1ll << 31)) return HL_ERR_UNSUPPORTED;
  if (r->n_tokens == 0) return HL_OK;
  st = rt_rows_ok(a, as, dim, es);
  return st != HL_OK ? st : rt_rows_ok(b, bs, dim, es);
}

template <class T>
static rt_geom rt_make_geom(const hl_route* r, int32_t dim) {
  const int parts = (dim + hl_vec<T>::N - 1) / hl_vec<T>::N;
  int lg = 0;
  while (lg < 8 && (1 << lg) < parts) ++lg;
  return {dim, r->k, lg, (parts + (1 << lg) - 1) >> lg, r->n_tokens, r->n_rows, r->n_experts};
}
#define RT_GRID_X (1u << 20)
static dim3 rt_grid(uint64_t blocks) {
  return blocks <= RT_GRID_X ? dim3((uint32_t)blocks) : dim3(RT_GRID_X, hl_div_up(blocks, RT_GRID_X));
}
// rows are whole cache lines
static bool rt_lines(const void* p, int64_t stride, int32_t dim, size_t es) {
  return ((uintptr_t)p | (uint64_t)stride * es | (uint64_t)dim * es) % HL_LINE == 0;
}
// KERNEL<T, UNI, KB ...>: the fewest rows in flight that hold a token's, so that no
// registers are kept for rows it does not have
#define RT_FORM(g, LAUNCH)                                         \
  do {                                                             \
    if ((g).lg >= 6) {                                             \
      if ((g).k <= 2) LAUNCH(true, 2);                             \
      else if ((g).k <= 4) LAUNCH(true, 4);                        \
      else LAUNCH(true, 8);                                        \
    } else {                                                       \
      if ((g).k <= 2) LAUNCH(false, 2);                            \
      else if ((g).k <= 4) LAUNCH(false, 4);                       \
      else LAUNCH(false, 8);                                       \
    }                                                              \
  } while (0)

extern "C" hl_status hl_route_plan(hl_handle* h, const hl_route* r, const int32_t* experts, void* workspace,
                                   size_t ws_bytes, hl_stream stream) {
  hl_status st = rt_check(h, r);
  if (st != HL_OK) return st;
  const int64_t n = r->n_tokens * r->k;
  if (n > 0 && !experts) return HL_ERR_INVALID_ARG;
  const int items = rt_items(n);
  const uint32_t tiles = rt_tile_count(n);
  if (tiles > 1 && (!workspace || (uintptr_t)workspace % 4 != 0)) return HL_ERR_INVALID_ARG;
  if (tiles > 1 && ws_bytes < hl_route_workspace_bytes(r->n_tokens, r->k, r->n_experts)) return HL_ERR_CAPACITY;
  hipStream_t s = (hipStream_t)stream;
  // (past the header, whose counters other calls on this workspace keep)
  hl_carver c = hl_carver::after_header(workspace, ws_bytes);
  uint32_t* hist = workspace ? c.take<uint32_t>(1) : nullptr;
  if (workspace) hl_ws_note(h, workspace, HL_WSK_OTHER);
  const int bits = r->n_experts > 1 ? hl_bit_width((uint64_t)r->n_experts - 1) : 0;
  const rt_shape sh = {(int32_t)n,  r->n_experts, bits, r->capacity ? r->capacity : INT32_MAX, r->align,
                       r->n_rows};
  const int mode = tiles == 1 ? 0 : ((int64_t)tiles * r->n_experts <= RT_DIRECT ? 1 : 2);
  const uint32_t cnt = (uint32_t)(RT_WAVES * r->n_experts * 2), lds = cnt + (uint32_t)(3 * r->n_experts + 1) * 4;
#define RT_PLAN(I)                                                                                                  \
  do {                                                                                                              \
    if (mode) HL_KERNEL(h, s, "rt_tiles", (rt_tiles<I>), dim3(tiles), dim3(RT_THREADS), cnt, s, experts, sh, hist, h->d_err); \
    if (mode == 2) HL_KERNEL(h, s, "rt_prefix", rt_prefix, dim3(r->n_experts), dim3(256), 0, s, hist, tiles, r->n_experts); \
    HL_KERNEL(h, s, "rt_place", (rt_place<I>), dim3(tiles), dim3(RT_THREADS), lds, s, experts, sh, (const uint32_t*)hist, \
              tiles, mode, r->counts, r->offsets, r->pos, r->order, h->d_err);                                      \
  } while (0)
  if (items == 1) RT_PLAN(1);
  else if (items == 2) RT_PLAN(2);
  else if (items == 4) RT_PLAN(4);
  else RT_PLAN(8);
#undef RT_PLAN
  HL_LAUNCHED();
  return HL_OK;
}

template <class T>
static void launch_gather(const hl_handle* h, const hl_route* r, int32_t dim, const void* x, int64_t xs, void* out,
                          int64_t os, hipStream_t s) {
  const rt_geom g = rt_make_geom<T>(r, dim);
  const uint32_t blocks = hl_div_up((uint64_t)g.n_tokens * g.chunks, 256 >> g.lg);
  const dim3 grid = rt_grid((uint64_t)blocks + (r->align > 1 ? r->n_experts : 0));
  const bool lines = rt_lines(out, os, dim, sizeof(T));
#define GATHER_(U, K, H)                                                                                            \
  HL_KERNEL(h, s, "rt_gather", (rt_gather<T, U, K, H>), grid, dim3(256), 0, s, g, blocks, r->pos, r->counts,        \
            r->offsets, (const T*)x, xs, (T*)out, os, h->d_err)
#define GATHER(U, K)            \
  do {                          \
    if (lines) GATHER_(U, K, true); \
    else GATHER_(U, K, false);  \
  } while (0)
  RT_FORM(g, GATHER);
#undef GATHER
#undef GATHER_
}

extern "C" hl_status hl_route_gather(const hl_handle* h, const hl_route* r, int32_t dtype, int32_t dim, const void* x,
                                     int64_t x_stride, void* rows, int64_t rows_stride, hl_stream stream) {
  hl_status st = rt_check_rows(h, r, dtype, dim, x, x_stride, rows, rows_stride);
  if (st != HL_OK || r->n_tokens == 0) return st;
  HL_BY_TYPE(dtype, launch_gather, h, r, dim, x, x_stride, rows, rows_stride, (hipStream_t)stream);
  HL_LAUNCHED();
  return HL_OK;
}

template <class T>
static void launch_combine(const hl_handle* h, const hl_route* r, int32_t dim, const void* rows, int64_t rs,
                           const float* weights, void* out, int64_t os, hipStream_t s) {
  const rt_geom g = rt_make_geom<T>(r, dim);
  const dim3 grid = rt_grid(hl_div_up((uint64_t)g.n_tokens * g.chunks, 256 >> g.lg));
  const bool lines = rt_lines(rows, rs, dim, sizeof(T));
#define COMBINE_(U, K, W, H)                                                                                        \
  HL_KERNEL(h, s, "rt_combine", (rt_combine<T, U, K, W, H>), grid, dim3(256), 0, s, g, r->pos, (const T*)rows, rs,   \
            weights, (T*)out, os, h->d_err)
#define COMBINE(U, K)                                       \
  do {                                                      \
    if (weights && lines) COMBINE_(U, K, true, true);       \
    else if (weights) COMBINE_(U, K, true, false);          \
    else if (lines) COMBINE_(U, K, false, true);            \
    else COMBINE_(U, K, false, false);                      \
  } while (0)
  RT_FORM(g, COMBINE);
#undef COMBINE_
#undef COMBINE
}

extern "C" hl_status hl_route_combine(const hl_handle* h, const hl_route* r, int32_t dtype, int32_t dim,
                                      const void* rows, int64_t rows_stride, const float* weights, void* out,
                                      int64_t out_stride, hl_stream stream) {
  hl_status st = rt_check_rows(h, r, dtype, dim, rows, rows_stride, out, out_stride);
  if (st != HL_OK || r->n_tokens == 0) return st;
  if ((uintptr_t)weights % 4 != 0) return HL_ERR_INVALID_ARG;
  HL_BY_TYPE(dtype, launch_combine, h, r, dim, rows, rows_stride, weights, out, out_stride, (hipStream_t)stream);
  HL_LAUNCHED();
  return HL_OK;
}

extern "C" hl_status hl_route_gather_bwd(const hl_handle* h, const hl_route* r, int32_t dtype, int32_t dim,
                                         const void* drows, int64_t drows_stride, void* dx, int64_t dx_stride,
                                         hl_stream stream) {
  return hl_route_combine(h, r, dtype, dim, drows, drows_stride, nullptr, dx, dx_stride, stream);
}

template <class T>
static void launch_combine_bwd(const hl_handle* h, const hl_route* r, int32_t dim, const void* dout, int64_t ds,
                               const void* rows, int64_t rs, const float* weights, void* drows, int64_t drs,
                               float* dweights, hipStream_t s) {
  rt_geom g = rt_make_geom<T>(r, dim);
  // (a row that leaves a fifth of its lanes idle: half of them, in two rounds; rows of 333 floats 28.9 us for
  // 30,000 assignments with a round, 26.4 with two; rows that fill their lanes lose by it: 30.0 and 34.6 for
  // 32,768 of 1024 bf16)
  if (g.lg > 6 && g.chunks == 1 && 5 * ((dim + hl_vec<T>::N - 1) / hl_vec<T>::N) <= 4 << g.lg) --g.lg;
  const uint32_t blocks = hl_div_up((uint64_t)g.n_tokens, 256 >> g.lg);
  const dim3 grid = rt_grid((uint64_t)blocks + (r->align > 1 ? r->n_experts : 0));
  const bool lines = rt_lines(rows, rs, g.dim, sizeof(T));
#define COMBINE_BWD_(U, K, H)                                                                                        \
  HL_KERNEL(h, s, "rt_combine_bwd", (rt_combine_bwd<T, U, K, H>), grid, dim3(256), 0, s, g, blocks, r->pos,          \
            r->counts, r->offsets, (const T*)dout, ds, (const T*)rows, rs, weights, (T*)drows, drs, dweights, h->d_err)
#define COMBINE_BWD(U, K)               \
  do {                                  \
    if (lines) COMBINE_BWD_(U, K, true); \
    else COMBINE_BWD_(U, K, false);     \
  } while (0)
  RT_FORM(g, COMBINE_BWD);
#undef COMBINE_BWD
#undef COMBINE_BWD_
}

extern "C" hl_status hl_route_combine_bwd(const hl_handle* h, const hl_route* r, int32_t dtype, int32_t dim,
                                          const void* dout, int64_t dout_stride, const void* rows, int64_t rows_stride,
                                          const float* weights, void* drows, int64_t drows_stride, float* dweights,
                                          hl_stream stream) {
  hl_status st = rt_check_rows(h, r, dtype, dim, dout, dout_stride, drows, drows_stride);
  if (st != HL_OK || r->n_tokens == 0) return st;
  if ((uintptr_t)weights % 4 != 0 || (uintptr_t)dweights % 4 != 0) return HL_ERR_INVALID_ARG;
  if (dweights && (st = rt_rows_ok(rows, rows_stride, dim, hl_elem_bytes(dtype))) != HL_OK) return st;
  HL_BY_TYPE(dtype, launch_combine_bwd, h, r, dim, dout, dout_stride, rows, rows_stride, weights, drows, drows_stride,
             dweights, (hipStream_t)stream);
  HL_LAUNCHED();
  return HL_OK;
}
