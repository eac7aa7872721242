// Which blocks of a paged cache a decode step reads.  A block's bounds are, per KV head and channel, the least and the largest
// key of its tokens, and its mass the sum of their degrees.  For a query q every token of the block has
//   q . k <= sum_d max(q_d lo_d, q_d hi_d),   so that   sum_t N_t exp(scale q . k_t) <= mass exp(scale sum_d max(q_d lo_d, q_d hi_d)):
// the logarithm of the right-hand side, the largest over the query heads of the KV head, is the block's score, and the blocks
// with the largest scores are the ones to read.
#include "ckv_internal.h"
#include "ckv_device.h"

namespace ckv {
namespace {

// x if it is less (more) than m or no number: one of a channel's keys that is none makes its bounds none
__device__ __forceinline__ float least(float m, float x) { return (x < m || x != x) ? x : m; }
__device__ __forceinline__ float most(float m, float x) { return (x > m || x != x) ? x : m; }

// one wave a (block, head); a lane takes a 16-byte piece of every row it sees
constexpr int kBoundsThreads = 256;
template <typename T>
__global__ __launch_bounds__(kBoundsThreads) void paged_bounds_kernel(const T* __restrict__ K, const int32_t* __restrict__ deg,
                                                                      PagedView paged, const int32_t* __restrict__ lens,
                                                                      const int32_t* __restrict__ since, int max_new, int heads,
                                                                      int dim, T* __restrict__ bounds, int32_t* __restrict__ mass) {
  constexpr int E = 16 / sizeof(T);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.z;
  const int h = blockIdx.y, bs = 1 << paged.shift;
  const int64_t row_tokens = (int64_t)paged.max_blocks << paged.shift;
  const int len = (int)min((int64_t)lens[b], row_tokens);
  const int from = since ? max(since[b], 0) : 0;
  const int to = (int)min((int64_t)len, (int64_t)from + max_new);
  const int col = (from >> paged.shift) + blockIdx.x * (kBoundsThreads / 64) + wave;
  if (from >= to || ((int64_t)col << paged.shift) >= to) return;
  const int blk = paged.table[(int64_t)b * paged.max_blocks + col];
  if ((unsigned)blk >= (unsigned)paged.n_blocks) return;
  const int n = min(bs, len - (col << paged.shift));
  const int pieces = dim / E, rows = 64 / pieces;        // (64 is a multiple of pieces)
  const int piece = lane % pieces;
  const int64_t slab = (int64_t)blk * heads + h;
  float lo[E], hi[E];
  int sum = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
  for (int t = lane / pieces; t < n; t += rows) {
    const int d = deg ? deg[(slab << paged.shift) + t] : 1;
    if (d < 1) continue;
    struct { T x[E]; } p;
    *reinterpret_cast<uint4*>(&p) = *reinterpret_cast<const uint4*>(K + ((slab << paged.shift) + t) * dim + piece * E);
#pragma unroll
    for (int e = 0; e < E; ++e) { lo[e] = least(lo[e], (float)p.x[e]); hi[e] = most(hi[e], (float)p.x[e]); }
    sum += d;
  }
  for (int w = pieces; w < 64; w *= 2) {
#pragma unroll
    for (int e = 0; e < E; ++e) { lo[e] = least(lo[e], __shfl_xor(lo[e], w)); hi[e] = most(hi[e], __shfl_xor(hi[e], w)); }
    sum += __shfl_xor(sum, w);
  }
  if (lane < pieces) {
    struct { T x[E]; } p, q;
#pragma unroll
    for (int e = 0; e < E; ++e) { p.x[e] = (T)lo[e]; q.x[e] = (T)hi[e]; }   // (exact: they are keys)
    T* to_p = bounds + slab * 2 * dim + piece * E;
    *reinterpret_cast<uint4*>(to_p) = *reinterpret_cast<const uint4*>(&p);
    *reinterpret_cast<uint4*>(to_p + dim) = *reinterpret_cast<const uint4*>(&q);
    if (lane == 0) mass[slab] = sum;
  }
}

// Ranks, largest first: a block that is always read, a score that is no finite fp32 number, the scores, a block without tokens
// that count or outside the pool.
constexpr uint32_t kAlways = 0xffffffffu, kNotFinite = 0xfffffffeu, kNothing = 0u;

// The score in 64 bits, rounded once to fp32.  In 32 bits the order of close scores would hang on the order of the sums, and
// neighbours at the cut are close: a selection among 2048 blocks has one chance in some hundred to come out differently.
__device__ __forceinline__ uint32_t rank_of(double dot, double scale, int mass) {
  const float s = (float)(dot * scale + log((double)mass));
  return (__float_as_uint(s) & 0x7f800000u) == 0x7f800000u ? kNotFinite : order_key(s);
}

// one wave a block: keys[b, h, block]
constexpr int kScoreThreads = 256;
template <typename T, int G>
__global__ __launch_bounds__(kScoreThreads) void paged_score_kernel(const T* __restrict__ q, const T* __restrict__ bounds,
                                                                    const int32_t* __restrict__ mass, PagedView paged,
                                                                    const int32_t* __restrict__ lens, int max_len, int heads, int dim,
                                                                    int n_select, int n_sink, int n_recent, float scale,
                                                                    uint32_t* __restrict__ keys, int key_stride) {
  const int lane = threadIdx.x & 63, b = blockIdx.z, h = blockIdx.y;
  const int n = div_up(max(min(lens[b], max_len), 0), 1 << paged.shift);
  const int i = blockIdx.x * (kScoreThreads / 64) + (threadIdx.x >> 6);
  if (i >= n || n <= n_select) return;
  uint32_t key = kNothing;
  const int blk = paged.table[(int64_t)b * paged.max_blocks + i];
  if (i < n_sink || i >= n - n_recent) key = kAlways;
  else if ((unsigned)blk < (unsigned)paged.n_blocks) {
    const int64_t slab = (int64_t)blk * heads + h;
    const int m = mass[slab];
    if (m > 0) {
      double best = -INFINITY;
      bool finite = true;
      for (int g = 0; g < G; ++g) {
        double x = 0.;
        for (int d = lane; d < dim; d += 64) {
          const double a = (double)(float)q[(((int64_t)b * heads + h) * G + g) * dim + d];
          x += fma(fmin(a, 0.), (double)(float)bounds[slab * 2 * dim + d], fmax(a, 0.) * (double)(float)bounds[(slab * 2 + 1) * dim + d]);
        }
        for (int w = 1; w < 64; w *= 2) x += __shfl_xor(x, w);
        finite = finite && x - x == 0.;
        best = fmax(best, x);
      }
      key = finite ? rank_of(best, (double)scale, m) : kNotFinite;
    }
  }
  if (lane == 0) keys[((int64_t)b * heads + h) * key_stride + i] = key;
}

// The n_select blocks of the largest keys of a (sequence, KV head), ties to the lower block, in ascending order.
constexpr int kSelectThreads = 256;
__device__ __forceinline__ int scan_int(int x, int* s_wave, int& all) {
  x = (int)wave_inclusive_scan((uint32_t)x);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 63) s_wave[wave] = x;
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < kSelectThreads / 64; ++w) {
    if (w == wave) before = all;
    all += s_wave[w];
  }
  __syncthreads();
  return x + before;
}
__global__ __launch_bounds__(kSelectThreads) void paged_select_kernel(const uint32_t* __restrict__ keys, int key_stride, PagedView paged,
                                                                      const int32_t* __restrict__ lens, int max_len, int heads,
                                                                      int n_select, int32_t* __restrict__ sel, int32_t* __restrict__ sel_lens) {
  __shared__ int s_hist[256], s_wave[kSelectThreads / 64], s_found[2];
  const int tid = threadIdx.x, h = blockIdx.x, b = blockIdx.y;
  const int len = max(min(lens[b], max_len), 0), bs = 1 << paged.shift, n = div_up(len, bs);
  const int64_t bh = (int64_t)b * heads + h;
  const uint32_t* key = keys + bh * key_stride;
  uint32_t cut = 0;              // every key above it is taken, and `ties` of those that equal it
  int ties = 0;
  if (n > n_select) {
    int want = n_select;
    uint32_t prefix = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      s_hist[tid] = 0;
      __syncthreads();
      for (int i = tid; i < n; i += kSelectThreads)
        if (shift == 24 || (key[i] >> (shift + 8)) == prefix) atomicAdd(&s_hist[(key[i] >> shift) & 255], 1);
      __syncthreads();
      int all;
      const int count = s_hist[255 - tid], upto = scan_int(count, s_wave, all);   // (digits in falling order)
      if (upto >= want && upto - count < want) { s_found[0] = 255 - tid; s_found[1] = want - (upto - count); }
      __syncthreads();
      prefix = (prefix << 8) | (uint32_t)s_found[0];
      want = s_found[1];
    }
    cut = prefix;
    ties = want;
  }
  int at = 0, tied = 0;
  for (int i0 = 0; i0 < n; i0 += kSelectThreads) {
    const int i = i0 + tid;
    const uint32_t x = n > n_select && i < n ? key[i] : 0u;
    bool in = i < n;
    if (n > n_select) {
      int all;
      const bool tie = in && x == cut;
      const int rank = tied + scan_int(tie, s_wave, all);
      tied += all;
      in = in && (x > cut || (tie && rank <= ties));
    }
    int all;
    const int place = at + scan_int(in, s_wave, all) - 1;
    at += all;
    if (in) {
      const int blk = paged.table[(int64_t)b * paged.max_blocks + i];
      sel[bh * n_select + place] = (unsigned)blk < (unsigned)paged.n_blocks ? blk * heads + h : -1;
    }
    if (i == n - 1) s_found[0] = in;
  }
  for (int i = at + tid; i < n_select; i += kSelectThreads) sel[bh * n_select + i] = -1;
  __syncthreads();
  if (tid == 0) sel_lens[bh] = n == 0 ? 0 : at * bs - (s_found[0] ? n * bs - len : 0);
}

template <typename T>
hipError_t launch_scores(int G, const SelectCall& c) {
  const dim3 grid((unsigned)div_up(c.key_stride, kScoreThreads / 64), (unsigned)c.heads, (unsigned)c.n_b);
#define CKV_SCORE(g)                                                                                                      \
  case g:                                                                                                                 \
    hipLaunchKernelGGL((paged_score_kernel<T, g>), grid, dim3(kScoreThreads), 0, c.st, static_cast<const T*>(c.q),         \
                       static_cast<const T*>(c.bounds), c.mass, c.paged, c.lens, c.max_len, c.heads, c.dim, c.n_select,    \
                       c.n_sink, c.n_recent, c.scale, c.keys, c.key_stride);                                               \
    break
  switch (G) {
    CKV_SCORE(1);
    CKV_SCORE(2);
    CKV_SCORE(4);
    CKV_SCORE(8);
    default: return hipErrorInvalidValue;
  }
#undef CKV_SCORE
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_bounds(const void* K, const int32_t* deg, int dtype, PagedView paged, const int32_t* lens, const int32_t* since,
                               int max_new, int n_b, int heads, int dim, void* bounds, int32_t* mass, hipStream_t st) {
  ScopedTimer t("paged_bounds", st);
  const int bs = 1 << paged.shift;
  // tokens [since, since + max_new) touch at most this many blocks
  const int64_t cols = ((int64_t)max_new + bs - 2) / bs + 1;
  const int n_cols = (int)(cols < paged.max_blocks ? cols : paged.max_blocks);
  const dim3 grid((unsigned)div_up(n_cols, kBoundsThreads / 64), (unsigned)heads, (unsigned)n_b);
  if (dtype == CKV_BF16)
    hipLaunchKernelGGL(paged_bounds_kernel<__bf16>, grid, dim3(kBoundsThreads), 0, st, static_cast<const __bf16*>(K), deg, paged, lens,
                       since, max_new, heads, dim, static_cast<__bf16*>(bounds), mass);
  else
    hipLaunchKernelGGL(paged_bounds_kernel<float>, grid, dim3(kBoundsThreads), 0, st, static_cast<const float*>(K), deg, paged, lens,
                       since, max_new, heads, dim, static_cast<float*>(bounds), mass);
  return hipGetLastError();
}

hipError_t launch_paged_select(int dtype, int G, const SelectCall& c) {
  {
    ScopedTimer t("paged_score", c.st);
    const hipError_t e = dtype == CKV_BF16 ? launch_scores<__bf16>(G, c) : launch_scores<float>(G, c);
    if (e != hipSuccess) return e;
  }
  ScopedTimer t("paged_select", c.st);
  hipLaunchKernelGGL(paged_select_kernel, dim3((unsigned)c.heads, (unsigned)c.n_b), dim3(kSelectThreads), 0, c.st, c.keys, c.key_stride,
                     c.paged, c.lens, c.max_len, c.heads, c.n_select, c.sel, c.sel_lens);
  return hipGetLastError();
}

}  // namespace ckv
