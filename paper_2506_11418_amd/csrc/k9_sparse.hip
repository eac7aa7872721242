// Which blocks of a paged cache a decode step reads.  A block's bounds are, per KV head and channel, the least and the largest
// key of its tokens, and its mass the sum of their degrees.  For a query q every token of the block has
//   q . k <= sum_d max(q_d lo_d, q_d hi_d),   so that   sum_t N_t exp(scale q . k_t) <= mass exp(scale sum_d max(q_d lo_d, q_d hi_d)):
// the logarithm of the right-hand side, the largest over the query heads of the KV head, is the block's score, and the blocks
// with the largest scores are the ones to read.
#include <type_traits>

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

// Ranks, largest first: a score that is no finite fp32 number, the scores, a block without tokens that count or outside the pool.
// No rank is 0xffffffff.
constexpr uint32_t kNotFinite = 0xfffffffeu, kNothing = 0u;

// The score in 64 bits, rounded once to fp32.  In 32 bits the order of close scores would hang on the order of the sums, and
// neighbours at the cut are close: a selection among 2048 blocks has one chance in some hundred to come out differently.
__device__ __forceinline__ uint32_t rank_of(double dot, double scale, int mass) {
  const float s = (float)(dot * scale + log((double)mass));
  return (__float_as_uint(s) & 0x7f800000u) == 0x7f800000u ? kNotFinite : order_key(s);
}

// Scores, 16 blocks a wave at a time, on the 64-bit matrix instruction that takes four products of 4x4 by 4x4 (A[i][k] of product p
// in lane i + 4p + 16k, B[k][j] in lane j + 4p + 16k, D[i][j] in lane j + 4p + 16i; checked on the GPU with whole numbers).
// Rows i + 4p are the blocks, columns the query heads, and the contraction runs over a block's bounds as they lie in
// memory, lo then hi: sum_d max(q_d lo_d, q_d hi_d) = sum_d min(q_d, 0) lo_d + max(q_d, 0) hi_d.  (Where that makes a NaN of zero
// and infinity the score is not finite either way.)  A 16-byte piece of a row goes to lane block + 16 (piece % 4), and the
// queries wait in fp32, as they are in 64 bits, in the order of the pieces.
//
// What bounds it: 16 cycles of the matrix unit and 12 of the vector unit (two conversions, one unpacking) for 64 bounds, 128
// bytes in bf16: 16 TB/s over the chip, so that memory decides.  One wave a block with vector arithmetic and sums over the lanes
// took 165 us for 100 MB.
template <typename T, int D, int G>
struct ScoreTile {
  static constexpr int E = 16 / sizeof(T);                 // bounds in a piece
  static constexpr int L = 2 * D / E / 4;                  // pieces of a lane
  static constexpr int SETS = G > 4 ? 2 : 1;               // of four heads
  static constexpr bool AHEAD = 4 * L * (2 + SETS * E / 4) <= 160;   // registers for the next tile while one is worked on
};
constexpr int kScoreThreads = 256, kScoreWaves = kScoreThreads / 64;
template <typename T, int D, int G>
__global__ __launch_bounds__(kScoreThreads, 2) void paged_score_kernel(const T* __restrict__ q, const T* __restrict__ bounds,
                                                                       const int32_t* __restrict__ mass, PagedView paged,
                                                                       const int32_t* __restrict__ lens, int max_len, int heads,
                                                                       int n_select, int n_sink, int n_recent, float scale,
                                                                       uint32_t* __restrict__ keys, int key_stride) {
  typedef ScoreTile<T, D, G> S;
  constexpr int E = S::E, L = S::L;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = blockIdx.y, b = blockIdx.z;
  const int n = div_up(max(min(lens[b], max_len), 0), 1 << paged.shift);
  const int lo = n_sink, hi = n - n_recent;                // the blocks to rank
  const int first = (lo / 16 + blockIdx.x * kScoreWaves + wave) * 16, step = gridDim.x * kScoreWaves * 16;
  if (n <= n_select || first >= hi) return;
  const int row = lane & 15, k = lane >> 4;
  const int32_t* table = paged.table + (int64_t)b * paged.max_blocks;

  struct Piece16 { T x[E]; };
  float qv[S::SETS][L][E];
#pragma unroll
  for (int s = 0; s < S::SETS; ++s)
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const int at = (4 * j + k) * E;
      const Piece16 p = *reinterpret_cast<const Piece16*>(q + (((int64_t)b * heads + h) * G + (s * 4 + (lane & 3)) % G) * D + at % D);
#pragma unroll
      for (int e = 0; e < E; ++e) qv[s][j][e] = at < D ? fminf((float)p.x[e], 0.f) : fmaxf((float)p.x[e], 0.f);
    }

  struct Tile {
    uint4 v[L];
    int mass;          // 0 for a block outside the pool
  };
  auto id_of = [&](int i0) { return table[min(i0 + row, hi - 1)]; };
  auto issue = [&](Tile& t, int blk) {
    const bool in = (unsigned)blk < (unsigned)paged.n_blocks;
    const int64_t slab = (int64_t)(in ? blk : 0) * heads + h;
    t.mass = mass[slab];
    const char* p = reinterpret_cast<const char*>(bounds + slab * (2 * D)) + k * 16;
#pragma unroll
    for (int j = 0; j < L; ++j) t.v[j] = ldg16_stream(p + j * 64);
    t.mass = in ? t.mass : 0;
  };
  auto work = [&](const Tile& t, int i0) {
    if constexpr (S::SETS == 2)                            // eight heads in 64 bits do not fit the registers: widened every time
#pragma unroll
      for (int s = 0; s < S::SETS; ++s)
#pragma unroll
        for (int j = 0; j < L; ++j)
#pragma unroll
          for (int e = 0; e < E; ++e) asm volatile("" : "+v"(qv[s][j][e]));
    double acc[S::SETS][2] = {};
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const uint32_t w[4] = {t.v[j].x, t.v[j].y, t.v[j].z, t.v[j].w};
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float x;
        if constexpr (E == 8) x = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
        else x = __uint_as_float(w[e]);
#pragma unroll
        for (int s = 0; s < S::SETS; ++s)
          acc[s][e & 1] = __builtin_amdgcn_mfma_f64_4x4x4f64((double)x, (double)qv[s][j][e], acc[s][e & 1], 0, 0, 0);
      }
    }
    auto finite = [](double x) { return x - x == 0. ? x : (double)INFINITY; };
    double best = finite(acc[0][0] + acc[0][1]);
    if constexpr (S::SETS == 2) best = fmax(best, finite(acc[1][0] + acc[1][1]));
    auto across = [&](auto ctrl) {                        // the heads: lanes of a quad
      const uint64_t u = __builtin_bit_cast(uint64_t, best);
      const uint32_t a = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, decltype(ctrl)::value, 0xF, 0xF, true);
      const uint32_t c = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), decltype(ctrl)::value, 0xF, 0xF, true);
      best = fmax(best, __builtin_bit_cast(double, (uint64_t)c << 32 | a));
    };
    across(std::integral_constant<int, 0xB1>{});
    across(std::integral_constant<int, 0x4E>{});
    const int out = (lane >> 4) + (lane & 12);             // the block of this lane's D
    const int m = __shfl(t.mass, out), i = i0 + out;
    const uint32_t key = m > 0 ? rank_of(best, (double)scale, m) : kNothing;
    if ((lane & 3) == 0 && i >= lo && i < hi) keys[((int64_t)b * heads + h) * key_stride + i] = key;
  };
  // table entries are read two tiles ahead, bounds one
  Tile ta, tb;
  int next = id_of(first + step);
  issue(ta, id_of(first));
  if constexpr (S::AHEAD) {
    for (int i0 = first;; i0 += 2 * step) {
      const int blk = next;
      next = id_of(i0 + 2 * step);
      if (i0 + step < hi) issue(tb, blk);
      work(ta, i0);
      if (i0 + step >= hi) break;
      const int blk2 = next;
      next = id_of(i0 + 3 * step);
      if (i0 + 2 * step < hi) issue(ta, blk2);
      work(tb, i0 + step);
      if (i0 + 2 * step >= hi) break;
    }
  } else {
    for (int i0 = first;;) {
      work(ta, i0);
      i0 += step;
      if (i0 >= hi) break;
      issue(ta, next);
      next = id_of(i0 + step);
    }
  }
}

// The n_select blocks of a (sequence, KV head) to read, in ascending order: the always selected ones and the largest keys of the
// others, ties to the lower block.  A thread holds KEYS keys (rows of more than that are read again for every step).
//
// The cut is found by histograms of kBins bins of equal width between the least and the largest key: then inside the bin that
// holds it, until that bin is wholly taken or is one key.  Scores lie close together in their exponents, so that
// digits from the top would put most of them into a few bins, whose counters are then bumped one lane at a time.
// Places follow from ballots: 64 neighbouring blocks are a word of a bit mask.
constexpr int kBins = 2048;
template <int THREADS>
__device__ __forceinline__ int scan_int(int x, int* s_wave, int& all) {
  x = (int)wave_inclusive_scan((uint32_t)x);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 63) s_wave[wave] = x;
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w == wave) before = all;
    all += s_wave[w];
  }
  __syncthreads();
  return x + before;
}
template <int THREADS, int KEYS>
__global__ __launch_bounds__(THREADS) void paged_select_kernel(const uint32_t* __restrict__ keys, int key_stride, PagedView paged,
                                                               const int32_t* __restrict__ lens, int max_len, int heads,
                                                               int n_select, int n_sink, int n_recent, int32_t* __restrict__ sel,
                                                               int32_t* __restrict__ sel_lens) {
  constexpr int W = THREADS / 64, SPAN = THREADS * KEYS, WORDS = SPAN / 64;
  __shared__ int s_hist[kBins], s_wave[W], s_found[3];
  __shared__ uint32_t s_range[2];
  __shared__ uint64_t s_mask[WORDS];
  __shared__ int s_before[WORDS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = blockIdx.x, b = blockIdx.y;
  const int len = max(min(lens[b], max_len), 0), bs = 1 << paged.shift, n = div_up(len, bs);
  const int64_t bh = (int64_t)b * heads + h;
  const uint32_t* key = keys + bh * key_stride;
  const int32_t* table = paged.table + (int64_t)b * paged.max_blocks;
  int32_t* out = sel + bh * n_select;
  auto put = [&](int place, int i) {
    const int blk = table[i];
    out[place] = (unsigned)blk < (unsigned)paged.n_blocks ? blk * heads + h : -1;
  };
  if (n <= n_select) {
    for (int i = tid; i < n_select; i += THREADS) {
      if (i < n) put(i, i);
      else out[i] = -1;
    }
    if (tid == 0) sel_lens[bh] = len;
    return;
  }
  const int lo_i = n_sink, hi_i = n - n_recent, spans = div_up(n, SPAN);
  uint32_t x[KEYS];
  auto load = [&](int span) {
#pragma unroll
    for (int j = 0; j < KEYS; ++j) {
      const int i = span * SPAN + j * THREADS + tid;
      x[j] = i >= lo_i && i < hi_i ? key[i] : 0u;
    }
  };
  auto ranked = [&](int span, int j) { const int i = span * SPAN + j * THREADS + tid; return i >= lo_i && i < hi_i; };
  // the range of the keys
  if (tid == 0) { s_range[0] = 0xffffffffu; s_range[1] = 0u; s_found[0] = 0; }
  __syncthreads();
  {
    uint32_t least_key = 0xffffffffu, most_key = 0u;
    for (int span = 0; span < spans; ++span) {
      load(span);
#pragma unroll
      for (int j = 0; j < KEYS; ++j)
        if (ranked(span, j)) { least_key = min(least_key, x[j]); most_key = max(most_key, x[j]); }
    }
    for (int w = 1; w < 64; w *= 2) {
      least_key = min(least_key, (uint32_t)__shfl_xor((int)least_key, w));
      most_key = max(most_key, (uint32_t)__shfl_xor((int)most_key, w));
    }
    if (lane == 0) { atomicMin(&s_range[0], least_key); atomicMax(&s_range[1], most_key); }
  }
  __syncthreads();
  uint32_t from = s_range[0], to = s_range[1];   // the cut lies in [from, to]; what is above `to` is taken
  int want = n_select - n_sink - n_recent;       // of the keys in it, counted from the top
  bool whole = false;                            // all of them
  if (want == 0) from = to = 0xffffffffu;        // (no key is that large)
  while (want > 0) {
    const uint32_t width = to - from;
    const int shift = width < kBins ? 0 : 32 - __clz(width) - 11;
    for (int i = tid; i < kBins; i += THREADS) s_hist[i] = 0;
    __syncthreads();
    for (int span = 0; span < spans; ++span) {
      if (spans > 1) load(span);
#pragma unroll
      for (int j = 0; j < KEYS; ++j)
        if (ranked(span, j) && x[j] >= from && x[j] <= to) atomicAdd(&s_hist[(x[j] - from) >> shift], 1);
    }
    __syncthreads();
    constexpr int PER = kBins / THREADS;         // a thread's bins, in falling order
    int count[PER], mine = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) { count[i] = s_hist[kBins - 1 - (tid * PER + i)]; mine += count[i]; }
    int upto = scan_int<THREADS>(mine, s_wave, all) - mine;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (upto < want && upto + count[i] >= want) { s_found[0] = kBins - 1 - (tid * PER + i); s_found[1] = want - upto; s_found[2] = count[i]; }
      upto += count[i];
    }
    __syncthreads();
    const uint32_t base = from + ((uint32_t)s_found[0] << shift);
    to = base + min(to - base, (1u << shift) - 1);
    from = base;
    want = s_found[1];
    whole = want == s_found[2];
    __syncthreads();                             // (s_found and s_hist are free again)
    if (whole || from == to) break;
  }
  // places: the blocks before a word of 64, and in it
  int at = 0, tied = 0;
  for (int span = 0; span < spans; ++span) {
    if (spans > 1) load(span);
    const int words = min(WORDS, div_up(n - span * SPAN, 64));
    auto places = [&](auto&& test, int& before_all) {      // s_mask and s_before of the blocks that pass the test
#pragma unroll
      for (int j = 0; j < KEYS; ++j) {
        const uint64_t m = __ballot(test(j));
        if (lane == 0) s_mask[j * W + wave] = m;
      }
      __syncthreads();
      for (int w0 = 0; w0 < words; w0 += THREADS) {
        const int w = w0 + tid;
        const int c = w < words ? __popcll(s_mask[w]) : 0;
        int all;
        const int upto = scan_int<THREADS>(c, s_wave, all);
        if (w < words) s_before[w] = before_all + upto - c;
        before_all += all;
      }
      __syncthreads();
    };
    auto place_of = [&](int j) { return s_before[j * W + wave] + (int)__popcll(s_mask[j * W + wave] & ((1ull << lane) - 1)); };
    uint64_t first_ties = ~0ull;                 // bit j: this thread's j-th key, if it equals the cut, is taken
    if (!whole) {
      places([&](int j) { return ranked(span, j) && x[j] == from; }, tied);
#pragma unroll
      for (int j = 0; j < KEYS; ++j)
        if (place_of(j) >= want) first_ties &= ~(1ull << j);
      __syncthreads();                           // (read before the next ones are written)
    }
    auto taken = [&](int j) {
      const int i = span * SPAN + j * THREADS + tid;
      return i < n && (i < lo_i || i >= hi_i || (whole ? x[j] >= from : x[j] > from || (x[j] == from && (first_ties >> j & 1))));
    };
    places(taken, at);
#pragma unroll
    for (int j = 0; j < KEYS; ++j)
      if (taken(j)) {
        const int i = span * SPAN + j * THREADS + tid;
        put(place_of(j), i);
        if (i == n - 1) s_found[0] = -1;
      }
    __syncthreads();
  }
  if (tid == 0) sel_lens[bh] = n_select * bs - (s_found[0] == -1 ? n * bs - len : 0);
}

template <typename T, int D, int G>
hipError_t launch_scores(const SelectCall& c) {
  // four waves a workgroup; as many workgroups as run at once (two a CU at least), as long as every wave has a tile
  const int tiles = div_up(c.key_stride, 16 * kScoreWaves), pairs = c.n_b * c.heads;
  const int fit = div_up(4 * cu_count(), pairs);
  hipLaunchKernelGGL((paged_score_kernel<T, D, G>), dim3((unsigned)(tiles < fit ? tiles : fit), (unsigned)c.heads, (unsigned)c.n_b),
                     dim3(kScoreThreads), 0, c.st, static_cast<const T*>(c.q), static_cast<const T*>(c.bounds), c.mass, c.paged, c.lens,
                     c.max_len, c.heads, c.n_select, c.n_sink, c.n_recent, c.scale, c.keys, c.key_stride);
  return hipGetLastError();
}
template <typename T, int D>
hipError_t launch_scores_g(int G, const SelectCall& c) {
  switch (G) {
    case 1: return launch_scores<T, D, 1>(c);
    case 2: return launch_scores<T, D, 2>(c);
    case 4: return launch_scores<T, D, 4>(c);
    case 8: return launch_scores<T, D, 8>(c);
  }
  return hipErrorInvalidValue;
}
template <int THREADS, int KEYS>
hipError_t launch_select(const SelectCall& c) {
  hipLaunchKernelGGL((paged_select_kernel<THREADS, KEYS>), dim3((unsigned)c.heads, (unsigned)c.n_b), dim3(THREADS), 0, c.st, c.keys, c.key_stride,
                     c.paged, c.lens, c.max_len, c.heads, c.n_select, c.n_sink, c.n_recent, c.sel, c.sel_lens);
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
  hipError_t e = hipErrorInvalidValue;
  if (c.key_stride > c.n_select) {     // (otherwise no sequence has a block to leave out)
    ScopedTimer t("paged_score", c.st);
    if (dtype == CKV_BF16) e = c.dim == 128 ? launch_scores_g<__bf16, 128>(G, c) : c.dim == 64 ? launch_scores_g<__bf16, 64>(G, c) : e;
    else e = c.dim == 128 ? launch_scores_g<float, 128>(G, c) : c.dim == 64 ? launch_scores_g<float, 64>(G, c)
           : c.dim == 32 ? launch_scores_g<float, 32>(G, c) : e;
    if (e != hipSuccess) return e;
  }
  ScopedTimer t("paged_select", c.st);
  if (c.key_stride <= 2048) return launch_select<256, 8>(c);
  if (c.key_stride <= 16384) return launch_select<1024, 16>(c);
  return launch_select<1024, 32>(c);
}

}  // namespace ckv
