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

// Bounds.  One wave a (block, head), the heads of a block side by side; a lane takes a 16-byte piece of every 64/PIECES-th row, four
// rows at a time.  Keys are compared as whole numbers of their own width, whose order is that of the numbers once the lower bits of
// negative ones are turned over: five instructions for two bf16 and their place in both bounds, where fp32 comparisons that
// keep NaN take 18.  A NaN lies beyond the infinity of its sign, so that it ends up in one of the two bounds; both become NaN then.
//
// What bounds it: reads.  402 MB of keys, 13 of degrees and 50 of bounds (8 sequences of up to 32768 tokens, 8 heads) take 86 us, 5.4 TB/s;
// with fp32 comparisons and the degrees waited for before the keys 122.
constexpr int kBoundsThreads = 256, kBoundsWaves = kBoundsThreads / 64;
template <typename T> struct Ordered;
template <> struct Ordered<__bf16> {     // two a word
  typedef __attribute__((ext_vector_type(2))) int16_t V;
  static constexpr uint32_t kLeast = 0x80008000u, kMost = 0x7fff7fffu;    // beyond every number
  static constexpr uint16_t kInf = 0x7f80u;
  static __device__ __forceinline__ uint32_t turned(uint32_t w) { return w ^ (__builtin_bit_cast(uint32_t, __builtin_bit_cast(V, w) >> (int16_t)15) & 0x7fff7fffu); }
  static __device__ __forceinline__ uint32_t lesser(uint32_t a, uint32_t b) { return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b))); }
  static __device__ __forceinline__ uint32_t greater(uint32_t a, uint32_t b) { return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b))); }
  // bounds in the cache's type from turned words: (inf, -inf) of no token, NaN in both where one of them is
  static __device__ __forceinline__ void finish(uint32_t& lo, uint32_t& hi, bool none) {
    lo = turned(lo);
    hi = turned(hi);
    uint32_t nan = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (((lo >> (16 * i)) & 0x7fffu) > kInf || ((hi >> (16 * i)) & 0x7fffu) > kInf) nan |= 0x7fc0u << (16 * i);
    if (none) { lo = 0x7f807f80u; hi = 0xff80ff80u; }
    else { lo |= nan; hi |= nan; }
  }
};
template <> struct Ordered<float> {
  static constexpr uint32_t kLeast = 0x80000000u, kMost = 0x7fffffffu;
  static __device__ __forceinline__ uint32_t turned(uint32_t w) { return w ^ ((uint32_t)((int32_t)w >> 31) & 0x7fffffffu); }
  static __device__ __forceinline__ uint32_t lesser(uint32_t a, uint32_t b) { return (uint32_t)min((int32_t)a, (int32_t)b); }
  static __device__ __forceinline__ uint32_t greater(uint32_t a, uint32_t b) { return (uint32_t)max((int32_t)a, (int32_t)b); }
  static __device__ __forceinline__ void finish(uint32_t& lo, uint32_t& hi, bool none) {
    lo = turned(lo);
    hi = turned(hi);
    const uint32_t nan = (lo & 0x7fffffffu) > 0x7f800000u || (hi & 0x7fffffffu) > 0x7f800000u ? 0x7fc00000u : 0u;
    if (none) { lo = 0x7f800000u; hi = 0xff800000u; }
    else { lo |= nan; hi |= nan; }
  }
};
template <typename T, int PIECES>
__global__ __launch_bounds__(kBoundsThreads) void paged_bounds_kernel(const T* __restrict__ K, const int32_t* __restrict__ deg,
                                                                      PagedView paged, const int32_t* __restrict__ lens,
                                                                      const int32_t* __restrict__ since, int max_new, int heads,
                                                                      T* __restrict__ bounds, int32_t* __restrict__ mass) {
  typedef Ordered<T> O;
  constexpr int E = 16 / sizeof(T), D = PIECES * E, ROWS = 64 / PIECES, U = 4;
  const int lane = threadIdx.x & 63, b = blockIdx.y, bs = 1 << paged.shift;
  const int unit = blockIdx.x * kBoundsWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = unit % heads;
  const int64_t row_tokens = (int64_t)paged.max_blocks << paged.shift;
  const int len = (int)min((int64_t)lens[b], row_tokens);
  const int from = since ? max(since[b], 0) : 0;
  const int to = (int)min((int64_t)len, (int64_t)from + max_new);
  const int col = (from >> paged.shift) + unit / heads;
  if (from >= to || ((int64_t)col << paged.shift) >= to) return;
  const int blk = paged.table[(int64_t)b * paged.max_blocks + col];
  if ((unsigned)blk >= (unsigned)paged.n_blocks) return;
  const int n = min(bs, len - (col << paged.shift));
  const int piece = lane % PIECES, mine = lane / PIECES;
  const int64_t slab = (int64_t)blk * heads + h;
  const T* rows = K + (slab << paged.shift) * D + piece * E;
  const int32_t* degrees = deg ? deg + (slab << paged.shift) : nullptr;
  uint32_t lo[4], hi[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) { lo[i] = O::kMost; hi[i] = O::kLeast; }
  int sum = 0;
  for (int t0 = 0; t0 < n; t0 += ROWS * U) {
    uint4 v[U];
    int d[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = min(t0 + u * ROWS + mine, n - 1);
      v[u] = ldg16_stream(rows + (int64_t)t * D);
      d[u] = degrees ? degrees[t] : 1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool counts = t0 + u * ROWS + mine < n && d[u] > 0;
      const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = O::turned(w[i]);
        lo[i] = O::lesser(lo[i], counts ? x : O::kMost);
        hi[i] = O::greater(hi[i], counts ? x : O::kLeast);
      }
      sum += counts ? d[u] : 0;
    }
  }
#pragma unroll
  for (int w = PIECES; w < 64; w *= 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = O::lesser(lo[i], (uint32_t)__shfl_xor((int)lo[i], w));
      hi[i] = O::greater(hi[i], (uint32_t)__shfl_xor((int)hi[i], w));
    }
    sum += __shfl_xor(sum, w);
  }
  if (lane < PIECES) {
#pragma unroll
    for (int i = 0; i < 4; ++i) O::finish(lo[i], hi[i], sum == 0);
    T* out = bounds + slab * 2 * D + piece * E;
    *reinterpret_cast<uint4*>(out) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    *reinterpret_cast<uint4*>(out + D) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    if (lane == 0) mass[slab] = sum;
  }
}

// Ranks, largest first: a score that is no finite fp32 number, the scores, a block without tokens that count or outside the pool.
// No rank is 0: that is no block at all.
constexpr uint32_t kNotFinite = 0xffffffffu, kNothing = 1u;

// The score in 64 bits, rounded once to fp32.  In 32 bits the order of close scores would hang on the order of the sums, and
// neighbours at the cut are close: a selection among 2048 blocks has one chance in some hundred to come out differently.
__device__ __forceinline__ uint32_t rank_of(double dot, double scale, int mass) {
  const float s = (float)(dot * scale + log((double)mass));
  return (__float_as_uint(s) & 0x7f800000u) == 0x7f800000u ? kNotFinite : order_key(s);
}

// Scores, 16 blocks a wave at a time, on the 64-bit matrix instruction that takes four products of 4x4 by 4x4 (A[i][k] of product p
// in lane i + 4p + 16k, B[k][j] in lane j + 4p + 16k, D[i][j] in lane j + 4p + 16i; checked on the GPU with whole numbers).
// Rows i + 4p are the blocks, columns the query heads, and the contraction runs over a block's bounds as they lie in
// memory, lo then hi: sum_d max(q_d lo_d, q_d hi_d) = sum_d min(q_d, 0) lo_d + max(q_d, 0) hi_d for finite numbers.  An infinity or a NaN
// in a bound or a query makes a product of the right-hand side one, and the score counts as not finite, also where the maximum
// on the left would be (q_d above zero, lo_d = -infinity, hi_d finite).  A 16-byte piece of a row goes to lane block + 16 (piece % 4), and the
// queries wait in fp32, as they are in 64 bits, in the order of the pieces.
//
// Why this instruction: the sums have to be in 64 bits (see rank_of), and it takes 16 cycles for 64 bounds and four heads where vector
// arithmetic takes 8 for each head, and leaves four lanes to compare instead of sums over sixteen (one wave a block with vector
// arithmetic: 100 MB 165 us, now 29).  The 16x16x4 form takes 64 cycles for sixteen columns, of which four or eight are heads.
//
// What bounds it: 268 MB (one sequence of 65536 blocks, 8 heads of 4) take 58 us, 4.6 TB/s.  Matrix unit busy 26 %, vector unit 37 % of the
// cycles (counted; they share the 64-bit arithmetic); the rest are waits for rows of 512 bytes in no order.  Neither
// more nor fewer waves help (two workgroups a CU 63 us, four 59, six 61), nor the queries held in 64 bits (60).
template <typename T, int D, int G>
struct ScoreTile {
  static constexpr int E = 16 / sizeof(T);                 // bounds in a piece
  static constexpr int PIECES = 2 * D / E;                 // of a block's row
  static constexpr int L = PIECES / 4;                     // of a lane
  static constexpr int SETS = G > 4 ? 2 : 1;               // of four heads
  static constexpr int BYTES = 16 * PIECES * 16;           // of a tile in LDS
  // byte offset of a piece of a tile's row in LDS: the XOR spreads the 16 rows of one piece column over all banks
  __device__ static int lds(int row, int piece) { return (row * PIECES + (piece ^ (row & 7))) << 4; }
};
constexpr int kScoreThreads = 256, kScoreWaves = kScoreThreads / 64;
// waves a SIMD: the queries of eight heads of 128 channels, or an fp32 tile of them, take the registers of two; both of four
template <typename T, int D, int G>
constexpr int score_waves() { return sizeof(T) * D * (G > 4 ? 2 : 1) >= 1024 ? 1 : sizeof(T) * D * (G > 4 ? 2 : 1) >= 512 ? 2 : 3; }
template <typename T, int D, int G>
__global__ __launch_bounds__(kScoreThreads, (score_waves<T, D, G>())) void paged_score_kernel(const T* __restrict__ q, const T* __restrict__ bounds,
                                                                       const int32_t* __restrict__ mass, PagedView paged,
                                                                       const int32_t* __restrict__ lens, int max_len, int heads,
                                                                       int n_select, int n_sink, int n_recent, float scale,
                                                                       uint32_t* __restrict__ keys, int key_stride) {
  typedef ScoreTile<T, D, G> S;
  constexpr int E = S::E, L = S::L;
  __shared__ __attribute__((aligned(16))) unsigned char s_tile[kScoreWaves * S::BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b = blockIdx.y;
  const int n = div_up(max(min(lens[b], max_len), 0), 1 << paged.shift);
  const int unit = blockIdx.x * kScoreWaves + wave, h = unit % heads, waves = gridDim.x * kScoreWaves / heads;   // of one head
  const int lo = n_sink, hi = n - n_recent;                // the blocks to rank
  const int first = (lo / 16 + unit / heads) * 16, step = waves * 16;
  if (n <= n_select || first >= hi || unit >= waves * heads) return;
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
      for (int e = 0; e < E; ++e) {
        const float x = (float)p.x[e];
        qv[s][j][e] = at < D ? __builtin_elementwise_minimum(x, 0.f) : __builtin_elementwise_maximum(x, 0.f);   // (a NaN stays one)
      }
    }

  unsigned char* tile = s_tile + wave * S::BYTES;
  struct Tile {
    uint4 v[L];
    int mass;          // of block `row`; 0 outside the pool
  };
  auto id_of = [&](int i0) { return table[min(i0 + row, hi - 1)]; };
  // whole rows, consecutive lanes consecutive pieces (lane block + 16 piece straight from memory takes a row of cache tags for every four
  // lanes: 268 MB 80 us, so 69), read once and not kept (with ordinary loads a whole pass of 88 us takes 201)
  auto issue = [&](Tile& t, int blk) {
    const bool in = (unsigned)blk < (unsigned)paged.n_blocks;
    const int slab = (in ? blk : 0) * heads + h;
    t.mass = mass[slab];
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const int at = 64 * j + lane;
      t.v[j] = ldg16_stream(bounds + (int64_t)__shfl(slab, at / S::PIECES) * (2 * D) + at % S::PIECES * E);
    }
    t.mass = in ? t.mass : 0;
  };
  auto stage = [&](const Tile& t) {
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const int at = 64 * j + lane;
      *reinterpret_cast<uint4*>(tile + S::lds(at / S::PIECES, at % S::PIECES)) = t.v[j];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // other lanes' pieces are read next (a wave's accesses to LDS are in order)
  };
  auto work = [&](int tile_mass, int i0) {
    // (held in 64 bits for the whole loop they would take a third wave's registers, or spill)
#pragma unroll
    for (int s = 0; s < S::SETS; ++s)
#pragma unroll
      for (int j = 0; j < L; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) asm volatile("" : "+v"(qv[s][j][e]));
    double acc[S::SETS][2] = {};
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const uint4 v = *reinterpret_cast<const uint4*>(tile + S::lds(row, 4 * j + k));
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
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
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
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
    const int m = __shfl(tile_mass, out), i = i0 + out;
    const uint32_t key = m > 0 ? rank_of(best, (double)scale, m) : kNothing;
    if ((lane & 3) == 0 && i >= lo && i < hi) keys[((int64_t)b * heads + h) * key_stride + i] = key;
  };
  // table entries are read two tiles ahead, bounds one
  Tile t;
  int next = id_of(first + step);
  issue(t, id_of(first));
  for (int i0 = first;; i0 += step) {
    const int m = t.mass;
    stage(t);
    if (i0 + step < hi) issue(t, next);
    next = id_of(i0 + 2 * step);
    work(m, i0);
    if (i0 + step >= hi) break;
  }
}

// The blocks of a (sequence, KV head) to read, in ascending order: the always selected ones and the largest keys of the others,
// ties to the lower block.  A thread holds KEYS keys (rows of more than that are read again for every step).
//
// The cut is found by histograms of kBins bins of equal width between the least and the largest key: then inside the bin that
// holds it, until that bin is wholly taken or is one key.  Scores lie close together in their exponents, so that
// digits from the top would put most of them into a few bins, whose counters are then bumped one lane at a time.
// Places follow from ballots: 64 neighbouring keys are a word of a bit mask.
//
// One CU takes half a microsecond for every instruction that 65536 keys need, so that long rows are cut into segments: a
// workgroup each finds the keys of its segment that can be among the largest, and one more takes the cut among those
// (65536 blocks of 8 heads, 256 of them: 49 us in one step, 20 in two launches: segments 7, the cut 13).  Short rows are bound by the
// chain of steps between barriers: 6.6 us for 129 blocks of 8 heads, 7.0 for 2048 of 128.
enum class Step { WHOLE, SEGMENT, JOIN };
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
template <int THREADS, int KEYS, Step STEP>
__global__ __launch_bounds__(THREADS) void paged_select_kernel(SelectCall c) {
  constexpr int W = THREADS / 64, SPAN = THREADS * KEYS, WORDS = SPAN / 64;
  __shared__ int s_hist[kBins], s_wave[W], s_found[3], s_end;     // s_end: the last block is taken
  __shared__ uint32_t s_range[2];
  __shared__ uint64_t s_mask[WORDS];
  __shared__ int s_before[WORDS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = blockIdx.x, b = blockIdx.y;
  const int64_t bh = (int64_t)b * c.heads + h;
  const int32_t* table = c.paged.table + (int64_t)b * c.paged.max_blocks;
  const int32_t* other = nullptr;                // JOIN: the blocks the keys belong to
  const uint32_t* key = c.keys + bh * c.key_stride;
  int row = c.key_stride;                        // readable keys
  if constexpr (STEP == Step::SEGMENT) {
    key += blockIdx.z * SPAN;
    row -= blockIdx.z * SPAN;
  }
  if constexpr (STEP == Step::JOIN) {
    key = c.kept + bh * c.segments * c.most * 2;
    other = reinterpret_cast<const int32_t*>(key) + c.segments * c.most;
    row = c.segments * c.most;
  }
  // The first span's keys, and what they stand for where there are few, are on their way before the length is known: what lies behind it
  // is read and not looked at.  No load is behind a branch.
  constexpr bool kFew = KEYS <= 8 && STEP != Step::SEGMENT;
  uint32_t x[KEYS];
  int entry[kFew ? KEYS : 1];
  auto load = [&](int span) {
#pragma unroll
    for (int j = 0; j < KEYS; ++j) x[j] = key[min(span * SPAN + j * THREADS + tid, row - 1)];
  };
  load(0);
  if constexpr (kFew) {
#pragma unroll
    for (int j = 0; j < KEYS; ++j) entry[j] = (STEP == Step::JOIN ? other : table)[min(j * THREADS + tid, row - 1)];
  }
  const int bs = 1 << c.paged.shift, len = max(min(c.lens[b], c.max_len), 0), n = div_up(len, bs);
  auto named = [&](int blk) { return (unsigned)blk < (unsigned)c.paged.n_blocks ? blk * c.heads + h : -1; };
  int32_t* out = c.sel + bh * c.n_select;
  if (n <= c.n_select) {
    if (STEP == Step::SEGMENT) return;
    for (int i = tid; i < c.n_select; i += THREADS) out[i] = i < n ? named(table[i]) : -1;
    if (tid == 0) c.sel_lens[bh] = len;
    return;
  }
  // which keys count: [lo, hi) of the row
  int lo = c.n_sink, hi = n - c.n_recent, want = c.n_select - c.n_sink - c.n_recent;
  if constexpr (STEP == Step::SEGMENT) {
    const int at = blockIdx.z * SPAN;
    if (at >= n) return;                         // (not looked at by the last step)
    lo = min(max(lo - at, 0), SPAN);
    hi = min(max(hi - at, lo), SPAN);
    want = min(want, hi - lo);
  }
  if constexpr (STEP == Step::JOIN) {
    lo = 0;
    hi = div_up(n, c.segment) * c.most;
  }
  const int spans = max(div_up(hi, SPAN), 1);
  auto counted = [&](int span) {                 // 0 for keys that do not count
#pragma unroll
    for (int j = 0; j < KEYS; ++j) {
      const int i = span * SPAN + j * THREADS + tid;
      x[j] = (unsigned)(i - lo) < (unsigned)(hi - lo) ? x[j] : 0u;
    }
  };
  counted(0);
  auto each_span = [&](auto&& f) __attribute__((always_inline)) {
    for (int span = 0; span < spans; ++span) {
      if (spans > 1) { load(span); counted(span); }
      f(span);
    }
  };
  // the range of the keys
  if (tid == 0) { s_range[0] = 0xffffffffu; s_range[1] = 0u; s_end = 0; s_found[0] = s_found[1] = s_found[2] = 0; }
  __syncthreads();
  {
    uint32_t least_key = 0xffffffffu, most_key = 0u;         // (of the key below: 0 becomes the largest)
    each_span([&](int) {
#pragma unroll
      for (int j = 0; j < KEYS; ++j) { least_key = min(least_key, x[j] - 1); most_key = max(most_key, x[j]); }
    });
    for (int w = 1; w < 64; w *= 2) {
      least_key = min(least_key, (uint32_t)__shfl_xor((int)least_key, w));
      most_key = max(most_key, (uint32_t)__shfl_xor((int)most_key, w));
    }
    if (lane == 0) { atomicMin(&s_range[0], least_key); atomicMax(&s_range[1], most_key); }
  }
  __syncthreads();
  uint32_t from = s_range[0] + 1, to = s_range[1];           // the cut lies in [from, to]; what is above `to` is taken
  bool whole = false;                            // all of them
  const bool none = want == 0;
  int left = want;                               // to be taken in [from, to], counted from the top
  for (int round = 0; left > 0 && round < 3; ++round) {       // (three digits of 11 bits: from == to then, whatever the keys)
    const uint32_t width = to - from;
    const int shift = width < kBins ? 0 : 32 - __clz(width) - 11;
    for (int i = tid; i < kBins; i += THREADS) s_hist[i] = 0;
    __syncthreads();
    each_span([&](int) {
#pragma unroll
      for (int j = 0; j < KEYS; ++j)
        if (x[j] - from <= width) atomicAdd(&s_hist[(x[j] - from) >> shift], 1);
    });
    __syncthreads();
    constexpr int PER = kBins / THREADS;         // a thread's bins, in falling order
    int count[PER], mine = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) { count[i] = s_hist[kBins - 1 - (tid * PER + i)]; mine += count[i]; }
    int upto = scan_int<THREADS>(mine, s_wave, all) - mine;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (upto < left && upto + count[i] >= left) { s_found[0] = kBins - 1 - (tid * PER + i); s_found[1] = left - upto; s_found[2] = count[i]; }
      upto += count[i];
    }
    __syncthreads();
    const uint32_t base = from + ((uint32_t)s_found[0] << shift);
    to = base + min(to - base, (1u << shift) - 1);
    from = base;
    left = s_found[1];
    whole = left == s_found[2];
    __syncthreads();                             // (s_found and s_hist are free again)
    if (whole || from == to) break;
  }
  // places: the keys taken before a word of 64, and in it
  int at = 0, tied = 0;
  each_span([&](int span) {
    const int words = min(WORDS, max(div_up(hi - span * SPAN, 64), 0));
    auto places = [&](auto&& test, int& before_all) {        // s_mask and s_before of the keys that pass the test
#pragma unroll
      for (int j = 0; j < KEYS; ++j) {
        const uint64_t m = __ballot(test(j));
        if (lane == 0) s_mask[j * W + wave] = m;
      }
      __syncthreads();
      for (int w0 = 0; w0 < words; w0 += THREADS) {
        const int w = w0 + tid;
        const int n_in = w < words ? __popcll(s_mask[w]) : 0;
        int all;
        const int upto = scan_int<THREADS>(n_in, s_wave, all);
        if (w < words) s_before[w] = before_all + upto - n_in;
        before_all += all;
      }
      __syncthreads();
    };
    auto place_of = [&](int j) { return s_before[j * W + wave] + (int)__popcll(s_mask[j * W + wave] & ((1ull << lane) - 1)); };
    if (!whole && !none) {                       // of the keys that equal the cut the first ones; the others count no longer
      places([&](int j) { return x[j] == from; }, tied);
#pragma unroll
      for (int j = 0; j < KEYS; ++j)
        if (x[j] == from && place_of(j) >= left) x[j] = 0;
      __syncthreads();                           // (read before the next ones are written)
    }
    auto taken = [&](int j) { return !none && x[j] >= from && x[j] != 0; };
    places(taken, at);
#pragma unroll
    for (int j = 0; j < KEYS; ++j)
      if (taken(j)) {
        const int i = span * SPAN + j * THREADS + tid, to_place = place_of(j);
        if (to_place >= want) continue;          // (never, unless another call writes this one's scratch)
        if constexpr (STEP == Step::SEGMENT) {
          uint32_t* kept = c.kept + (bh * c.segments * 2 + blockIdx.z) * c.most + to_place;
          kept[0] = x[j];
          kept[c.segments * c.most] = (uint32_t)(blockIdx.z * SPAN + i);
        } else {
          int blk = entry[kFew ? j : 0];
          if (!kFew || spans > 1) blk = STEP == Step::JOIN ? other[i] : table[i];
          if ((STEP == Step::JOIN ? blk : i) == n - 1) s_end = 1;
          out[c.n_sink + to_place] = named(STEP == Step::JOIN ? table[blk] : blk);
        }
      }
    __syncthreads();
  });
  if constexpr (STEP == Step::SEGMENT) {
    uint32_t* kept = c.kept + (bh * c.segments * 2 + blockIdx.z) * c.most;
    for (int i = at + tid; i < c.most; i += THREADS) kept[i] = 0u;
  } else {
    for (int i = tid; i < c.n_sink + c.n_recent; i += THREADS) {
      const int place = i < c.n_sink ? i : i - c.n_sink + c.n_select - c.n_recent;
      out[place] = named(table[i < c.n_sink ? i : i - c.n_sink + n - c.n_recent]);
    }
    if (tid == 0) c.sel_lens[bh] = c.n_select * bs - (c.n_recent > 0 || s_end ? n * bs - len : 0);   // (the last block may be short)
  }
}

template <typename T, int D, int G>
hipError_t launch_scores(const SelectCall& c) {
  // Three workgroups a CU, as long as each wave has a tile; and whole heads, so that the rows of a block that lie side by side are
  // read together (a head a workgroup: 268 MB 67 us).  Three is what runs at once of most instances; of those with fewer
  // waves a SIMD (see score_waves) the rest is a second round (bf16, 128 channels, 61 x 8 heads of 8: 854 workgroups on 512 places).
  // Every sequence gets the same number, whatever its length.
  const int tiles = div_up(c.key_stride, 16), fit = div_up(3 * kScoreWaves * cu_count(), c.n_b * c.heads);
  const int waves = (tiles < fit ? tiles : fit) * c.heads;
  hipLaunchKernelGGL((paged_score_kernel<T, D, G>), dim3((unsigned)div_up(waves, kScoreWaves), (unsigned)c.n_b),
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
template <int THREADS, int KEYS, Step STEP>
hipError_t launch_select(const SelectCall& c) {
  hipLaunchKernelGGL((paged_select_kernel<THREADS, KEYS, STEP>), dim3((unsigned)c.heads, (unsigned)c.n_b, (unsigned)(STEP == Step::SEGMENT ? c.segments : 1)),
                     dim3(THREADS), 0, c.st, c);
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
  const dim3 grid((unsigned)(((int64_t)n_cols * heads + kBoundsWaves - 1) / kBoundsWaves), (unsigned)n_b);
#define CKV_BOUNDS(T, pieces)                                                                                               \
  hipLaunchKernelGGL((paged_bounds_kernel<T, pieces>), grid, dim3(kBoundsThreads), 0, st, static_cast<const T*>(K), deg, paged, lens, \
                     since, max_new, heads, static_cast<T*>(bounds), mass)
  const int pieces = dim * (dtype == CKV_BF16 ? 2 : 4) / 16;
  if (dtype == CKV_BF16 && pieces == 8) CKV_BOUNDS(__bf16, 8);
  else if (dtype == CKV_BF16 && pieces == 16) CKV_BOUNDS(__bf16, 16);
  else if (dtype == CKV_F32 && pieces == 8) CKV_BOUNDS(float, 8);
  else if (dtype == CKV_F32 && pieces == 16) CKV_BOUNDS(float, 16);
  else if (dtype == CKV_F32 && pieces == 32) CKV_BOUNDS(float, 32);
  else return hipErrorInvalidValue;
#undef CKV_BOUNDS
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
  SelectCall s = c;
  s.segment = kSelectSegment;
  s.segments = div_up(c.key_stride, kSelectSegment);
  s.most = c.n_select - c.n_sink - c.n_recent;
  s.kept = c.keys + (int64_t)c.n_b * c.heads * c.key_stride;
  ScopedTimer t("paged_select", c.st);
  // Threads and keys a thread, us on both sides of a border.  The last step of a row in segments, 512 x 8 / 1024 x 16: 2560 keys 7.5 /
  // 10.2, 4096 8.4 / 10.8, 8192 16.7 / 12.6.  Whole rows, 256 x 8 / 1024 x 8: 1024 keys of 128 rows 6.1 / 7.7, 2048 7.0 / 7.8, 2304
  // 10.5 / 8.0; 1024 x 8 / 1024 x 16: 4 x 8 rows of 8192 keys 8.8 / 11.0, 8 rows of 10000 14.7 / 11.5, of 16000 16.4 / 12.8.
  if (select_in_segments(c.key_stride, s.most)) {
    e = launch_select<256, kSelectSegment / 256, Step::SEGMENT>(s);
    if (e != hipSuccess) return e;
    return s.segments * s.most <= 4096 ? launch_select<512, 8, Step::JOIN>(s) : launch_select<1024, 16, Step::JOIN>(s);
  }
  if (c.key_stride <= 2048) return launch_select<256, 8, Step::WHOLE>(s);
  if (c.key_stride <= 8192) return launch_select<1024, 8, Step::WHOLE>(s);
  return launch_select<1024, 16, Step::WHOLE>(s);
}

}  // namespace ckv
