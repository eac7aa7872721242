// Rows of a block table forked and blocks moved: which block a page goes to is settled on the table and the free list (see
// k8_tables.hip for its layout), and the pages of every pool that shares them are then copied by the list of pairs.
//
// Tables and lists are small: what their kernels take is launches and waits for loads that depend on each other (3.5 to 6.5 us each, of the
// 12 to 13.5 us of a prompt of 500 tokens forked, copied and dropped again).  The copy is bound by memory.
#include "ckv_internal.h"
#include "ckv_device.h"

namespace ckv {
namespace {

constexpr int kListHead = 4;
constexpr int kInUse = INT32_MAX;
constexpr int kThreads = 256, kWaves = kThreads / 64;

__device__ __forceinline__ int blocks_of(int tokens, int shift) { return (tokens >> shift) + ((tokens & ((1 << shift) - 1)) != 0); }
// entries of a row that hold tokens
__device__ __forceinline__ int entries_of(int len, int max_blocks, int shift) { return min(blocks_of(max(len, 0), shift), max_blocks); }

// Sum of x over the threads before this one; `all` receives that over the whole workgroup.  s_wave: one word a wave.
template <int THREADS>
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t* s_wave, uint32_t& all) {
  const uint32_t upto = wave_inclusive_scan(x);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 63) s_wave[wave] = upto;
  __syncthreads();
  uint32_t before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w == wave) before = all;
    all += s_wave[w];
  }
  __syncthreads();
  return before + upto - x;
}

// ---- fork ----------------------------------------------------------------------------------------
// blocks among entries of a row, summed over a wave's lanes by the caller
template <int STEP>
__device__ __forceinline__ int blocks_among(const int32_t* row, int entries, int n_blocks, int first) {
  constexpr int kAhead = 4;                // loads in flight
  int count = 0;
  for (int j0 = first; j0 < entries; j0 += STEP * kAhead) {
    int id[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) id[i] = j0 + i * STEP < entries ? row[j0 + i * STEP] : -1;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) count += (unsigned)id[i] < (unsigned)n_blocks;
  }
  return count;
}
__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int w = 1; w < 64; w *= 2) x += __shfl_xor(x, w);
  return x;
}
// tokens of the row that row b continues, -1 where none is asked for or it cannot be
__device__ __forceinline__ int continued(const int32_t* lens, const int32_t* source, int b, int n_b, int max_blocks, int shift) {
  const int f = source[b];
  if ((unsigned)f >= (unsigned)n_b || f == b || lens[b] != 0) return -1;
  const int len = lens[f];
  return len >= 0 && len <= (int64_t)max_blocks << shift ? len : -1;
}

// need[b] := blocks of the row that row b continues, -1 where none is asked for or it cannot be.
__global__ __launch_bounds__(kThreads) void fork_count_kernel(const int32_t* __restrict__ table, const int32_t* __restrict__ lens,
                                                              const int32_t* __restrict__ source, int n_b, int max_blocks, int n_blocks, int shift,
                                                              int32_t* __restrict__ need) {
  __shared__ int s_count[kWaves];
  const int b = blockIdx.x, tid = threadIdx.x, len = continued(lens, source, b, n_b, max_blocks, shift);
  int count = 0;
  if (len > 0) count = blocks_among<kThreads>(table + (int64_t)source[b] * max_blocks, blocks_of(len, shift), n_blocks, tid);
  count = wave_sum(count);
  if ((tid & 63) == 0) s_count[tid >> 6] = count;
  __syncthreads();
  if (tid == 0) need[b] = len < 0 ? -1 : s_count[0] + s_count[1] + s_count[2] + s_count[3];
}

// Up to kRowsHere rows of kEntriesHere entries together are counted by the workgroups that deal, two rows a wave; else a launch of its own
// counts.  Replayed by a graph, with the two copies that restore the arguments, us here / by a launch: 2 rows of 32 8.7 / 10.1, 8 of 128
// 10.0 / 10.8, 16 of 64 10.9 / 10.6, 64 of 128 21.2 / 11.5; 155 of 3, by themselves, 31 / 11.
constexpr int kRowsHere = 8, kEntriesHere = 1024;
// Every workgroup sums the rows' needs for itself and deals to its share of the rows; the last one to arrive writes what the others
// have read: lengths, grants (which held the needs) and the number of free blocks.
// dynamic LDS: 8 bytes a row
template <int ROWS>   // rows of a thread's sums
__global__ __launch_bounds__(kThreads) void fork_deal_kernel(int32_t* __restrict__ table, int32_t* __restrict__ lens,
                                                             const int32_t* __restrict__ source, int32_t* __restrict__ free_list, int n_b,
                                                             int max_blocks, int n_blocks, int shift, int32_t* __restrict__ moves, int n_moves,
                                                             int32_t* __restrict__ granted, bool counted) {
  constexpr int kEach = 4;                 // entries of a row to a thread at a time
  extern __shared__ int32_t s_end[];
  int32_t* s_need = s_end + n_b;
  __shared__ uint32_t s_wave[kWaves];
  __shared__ int s_last, s_take;
  const int tid = threadIdx.x;
  const int n_free = min(max(free_list[0], 0), n_blocks), most = min(n_free, n_moves);
  const int32_t* stack = free_list + kListHead;
  int32_t* marks = free_list + kListHead + n_blocks;
  if (counted) {
    for (int b = tid; b < n_b; b += kThreads) s_need[b] = granted[b];
  } else {                                 // each workgroup counts them all, a row a wave
    for (int b = tid >> 6; b < n_b; b += kWaves) {
      const int len = continued(lens, source, b, n_b, max_blocks, shift);
      int count = len;
      if (len > 0) count = wave_sum(blocks_among<64>(table + (int64_t)source[b] * max_blocks, blocks_of(len, shift), n_blocks, tid & 63));
      if ((tid & 63) == 0) s_need[b] = count;
    }
  }
  if (tid == 0) s_take = 0;
  __syncthreads();
  int need[ROWS];
  uint32_t mine = 0, all;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    need[r] = tid * ROWS + r < n_b ? max(s_need[tid * ROWS + r], 0) : 0;
    mine += need[r];
  }
  uint32_t end = sum_before<kThreads>(mine, s_wave, all);
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    end += need[r];
    if (tid * ROWS + r < n_b) s_end[tid * ROWS + r] = (int)end;
    if (need[r] > 0 && end <= (uint32_t)most) atomicMax(&s_take, (int)end);
  }
  __syncthreads();
  const int take = s_take;
  for (int b = blockIdx.x; b < n_b; b += gridDim.x) {
    const int base = b ? s_end[b - 1] : 0;
    if (s_need[b] < 0 || (s_end[b] > base && s_end[b] > most)) continue;   // not asked for, or refused
    const int f = source[b], entries = blocks_of(lens[f], shift);
    const int32_t* from = table + (int64_t)f * max_blocks;
    int32_t* to = table + (int64_t)b * max_blocks;
    int dealt = base;
    for (int j0 = 0; j0 < entries; j0 += kThreads * kEach) {
      const int j = j0 + tid * kEach;
      int id[kEach];
      uint32_t real = 0, here;
#pragma unroll
      for (int i = 0; i < kEach; ++i) id[i] = j + i < entries ? from[j + i] : -1;
#pragma unroll
      for (int i = 0; i < kEach; ++i) real += (unsigned)id[i] < (unsigned)n_blocks;
      int at = dealt + (int)sum_before<kThreads>(real, s_wave, here);
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        int fresh = id[i];
        if ((unsigned)id[i] < (unsigned)n_blocks) {
          if (at < s_end[b]) {
            fresh = stack[n_free - 1 - at];
            moves[2 * at] = id[i];
            moves[2 * at + 1] = fresh;
            if ((unsigned)fresh < (unsigned)n_blocks) marks[fresh] = kInUse;
          }
          ++at;
        }
        if (j + i < entries) to[j + i] = fresh;
      }
      dealt += (int)here;
    }
  }
  for (int64_t i = 2 * (int64_t)take + blockIdx.x * kThreads + tid; i < 2 * (int64_t)n_moves; i += (int64_t)gridDim.x * kThreads) moves[i] = -1;
  __syncthreads();                         // (what this workgroup read has arrived: it has been stored or compared)
  if (tid == 0) s_last = gridDim.x == 1 || atomicAdd(&free_list[1], 1) == (int)gridDim.x - 1;
  __syncthreads();
  if (!s_last) return;
  // A row that is itself asked for was empty: what continues it is so too, whatever it becomes in this call.
  int len[ROWS], ok[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int b = tid + r * kThreads;
    len[r] = ok[r] = 0;
    if (b < n_b) {
      const int asked = s_need[b];
      ok[r] = asked == 0 || (asked > 0 && s_end[b] <= most);
      if (ok[r] && s_need[source[b]] < 0) len[r] = lens[source[b]];
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int b = tid + r * kThreads;
    if (b < n_b) {
      if (len[r] > 0) lens[b] = len[r];
      granted[b] = ok[r];
    }
  }
  if (tid == 0) {
    free_list[0] = n_free - take;
    if (gridDim.x > 1) atomicExch(&free_list[1], 0);
  }
}

// ---- compact -------------------------------------------------------------------------------------
// Two bits a block, in words of 32: free, and named by the table (and not free); before each word, how many of either.  With them
// everything is a matter of counting: the k highest of the table's blocks move into the k lowest free ones, k as large as leaves every
// one lower than it was.
struct CompactBits {
  uint32_t *free, *used, *free_before, *used_before;
};
struct CompactScratch {
  CompactBits bits;
  int32_t* head;                           // k, free blocks, the table's blocks
  uint8_t* named;                          // a byte a block, in 32 bytes a word
};

__device__ __forceinline__ uint32_t upto_bit(uint32_t word, int bit) { return word & ((1u << bit) - 1); }

// The largest k of which the words from `first` on, STEP apart, know: free ones below a block rise, the table's from there on fall, and
// the largest minimum of the two lies where they cross.
template <int STEP>
__device__ __forceinline__ int largest_k(const CompactBits& w, int words, int n_used, int first) {
  int k = 0;
  for (int i = first; i < words; i += STEP) {
    uint32_t below = w.free_before[i], above = n_used - w.used_before[i];
    const uint32_t f = w.free[i], u = w.used[i];
    k = max(k, (int)min(below, above));
    if (below < above && below + __popc(f) >= above - __popc(u))
      for (int bit = 0; bit < 32; ++bit) {
        below += (f >> bit) & 1;
        above -= (u >> bit) & 1;
        k = max(k, (int)min(below, above));
      }
  }
  return k;
}

// What block x becomes: moves, marks and the stack of free blocks, the lowest of them dealt first; whether it holds tokens then.
__device__ __forceinline__ bool settle(int x, const CompactBits& w, int k, int n_free, int n_used, int32_t* stack, int32_t* marks, int32_t* moves) {
  const int i = x >> 5, bit = x & 31;
  const uint32_t f = w.free[i], u = w.used[i];
  const int free_below = (int)(w.free_before[i] + __popc(upto_bit(f, bit))), used_below = (int)(w.used_before[i] + __popc(upto_bit(u, bit)));
  const int moved_below = max(used_below - (n_used - k), 0);              // the k highest move
  const bool home = ((f >> bit) & 1) && free_below < k, mover = ((u >> bit) & 1) && used_below >= n_used - k;
  if (home) {
    moves[2 * free_below + 1] = x;
    marks[x] = kInUse;
  }
  if (mover) {
    moves[2 * moved_below] = x;
    marks[x] = -1;
  }
  const bool free_now = mover || (((f >> bit) & 1) && !home);
  if (free_now) stack[n_free - 1 - (free_below - min(free_below, k) + moved_below)] = x;
  if (x >= n_free) stack[x] = -1;
  return !free_now;
}

// An entry's block after the moves.
__device__ __forceinline__ int renamed(int id, const CompactBits& w, int k, int n_used, const int32_t* moves) {
  const uint32_t u = w.used[id >> 5];
  const int above = n_used - (int)(w.used_before[id >> 5] + __popc(upto_bit(u, id & 31)));
  return ((u >> (id & 31)) & 1) && above <= k ? moves[2 * (k - above) + 1] : id;
}

__global__ __launch_bounds__(kThreads) void compact_free_kernel(const int32_t* __restrict__ free_list, int n_blocks, CompactScratch w,
                                                                int32_t* __restrict__ extent) {
  const int x = blockIdx.x * kThreads + threadIdx.x;
  const int32_t* marks = free_list + kListHead + n_blocks;
  const uint64_t bits = __ballot(x < n_blocks && marks[min(x, n_blocks - 1)] == -1);
  if ((threadIdx.x & 31) == 0 && x < n_blocks) w.bits.free[x >> 5] = (threadIdx.x & 32) ? (uint32_t)(bits >> 32) : (uint32_t)bits;
  if (x < div_up(n_blocks, 32) * 32) w.named[x] = 0;
  if (x == 0) *extent = 0;
}

__global__ __launch_bounds__(kThreads) void compact_used_kernel(const int32_t* __restrict__ table, const int32_t* __restrict__ lens, int max_blocks,
                                                                int n_blocks, int shift, CompactScratch w) {
  const int b = blockIdx.x, entries = entries_of(lens[b], max_blocks, shift);
  const int32_t* row = table + (int64_t)b * max_blocks;
  for (int j = blockIdx.y * kThreads + threadIdx.x; j < entries; j += gridDim.y * kThreads) {
    const int id = row[j];
    if ((unsigned)id < (unsigned)n_blocks) w.named[id] = 1;
  }
}

constexpr int kScanThreads = 1024;
// Counts before each word; returns the sums over all words.  used(i, free): a word's second bits.
template <typename Used>
__device__ __forceinline__ void count_words(const CompactBits& w, int words, uint32_t* s_wave, Used&& used, uint32_t& n_free, uint32_t& n_used) {
  n_free = n_used = 0;
  for (int w0 = 0; w0 < words; w0 += kScanThreads) {
    const int i = w0 + threadIdx.x;
    const uint32_t f = i < words ? w.free[i] : 0, u = i < words ? used(i, f) : 0;
    uint32_t all;
    const uint32_t f_before = sum_before<kScanThreads>(__popc(f), s_wave, all) + n_free;
    n_free += all;
    const uint32_t u_before = sum_before<kScanThreads>(__popc(u), s_wave, all) + n_used;
    n_used += all;
    if (i < words) {
      w.used[i] = u;
      w.free_before[i] = f_before;
      w.used_before[i] = u_before;
    }
  }
}

// a byte of 0 or 1 each into the bits of a word
__device__ __forceinline__ uint32_t bits_of(const uint8_t* named) {
  const uint4 a = *reinterpret_cast<const uint4*>(named), b = *reinterpret_cast<const uint4*>(named + 16);
  const uint32_t q[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint32_t u = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) u |= ((q[i] * 0x10204080u) >> 28) << (4 * i);
  return u;
}

__global__ __launch_bounds__(kScanThreads) void compact_scan_kernel(int words, int n_moves, CompactScratch w) {
  __shared__ uint32_t s_wave[kScanThreads / 64];
  __shared__ int s_k;
  const int tid = threadIdx.x;
  uint32_t n_free, n_used;
  if (tid == 0) s_k = 0;
  count_words(w.bits, words, s_wave, [&](int i, uint32_t f) { return bits_of(w.named + (int64_t)i * 32) & ~f; }, n_free, n_used);
  __syncthreads();                         // (a thread reads the words that it has written)
  const int k = largest_k<kScanThreads>(w.bits, words, (int)n_used, tid);
  if (k) atomicMax(&s_k, k);
  __syncthreads();
  if (tid == 0) {
    w.head[0] = min(s_k, n_moves);
    w.head[1] = (int)n_free;
    w.head[2] = (int)n_used;
  }
}

__global__ __launch_bounds__(kThreads) void compact_blocks_kernel(int32_t* __restrict__ free_list, int n_blocks, CompactScratch w,
                                                                  int32_t* __restrict__ moves, int n_moves, int32_t* __restrict__ extent) {
  const int x = blockIdx.x * kThreads + threadIdx.x;
  const int k = w.head[0], n_free = w.head[1], n_used = w.head[2];
  int32_t* stack = free_list + kListHead;
  const bool taken = x < n_blocks && settle(x, w.bits, k, n_free, n_used, stack, stack + n_blocks, moves);
  const uint64_t some = __ballot(taken);
  if (some && (threadIdx.x & 63) == 0) atomicMax(extent, x + 64 - (int)__builtin_clzll(some));
  for (int64_t i = 2 * (int64_t)k + x; i < 2 * (int64_t)n_moves; i += (int64_t)gridDim.x * kThreads) moves[i] = -1;
  if (x == 0) free_list[0] = n_free;
}

__global__ __launch_bounds__(kThreads) void compact_rename_kernel(int32_t* __restrict__ table, const int32_t* __restrict__ lens, int max_blocks,
                                                                  int n_blocks, int shift, CompactScratch w, const int32_t* __restrict__ moves) {
  const int b = blockIdx.x, entries = entries_of(lens[b], max_blocks, shift), k = w.head[0], n_used = w.head[2];
  int32_t* row = table + (int64_t)b * max_blocks;
  if (k == 0) return;
  for (int j = blockIdx.y * kThreads + threadIdx.x; j < entries; j += gridDim.y * kThreads) {
    const int id = row[j];
    if ((unsigned)id >= (unsigned)n_blocks) continue;
    const int now = renamed(id, w.bits, k, n_used, moves);
    if (now != id) row[j] = now;
  }
}

// The five steps in one workgroup, with the words in LDS.  Five launches, replayed by a graph, take 10 to 13 us up to 16384 blocks; this one
// 3.9 us for 128 entries and 256 blocks, 6.8 for 4096 and 4096, 10.2 for 8192 and 8192 (the five: 9.4, 10.7, 11.8), 17 for 16384 and 16384
// (13).
constexpr int kSmallBlocks = 8192, kSmallEntries = 8192;
__global__ __launch_bounds__(kScanThreads) void compact_small_kernel(int32_t* __restrict__ table, const int32_t* __restrict__ lens,
                                                                     int32_t* __restrict__ free_list, int n_b, int max_blocks, int n_blocks, int shift,
                                                                     int32_t* __restrict__ moves, int n_moves, int32_t* __restrict__ extent) {
  constexpr int kWords = kSmallBlocks / 32;
  __shared__ uint32_t s_bits[4][kWords], s_wave[kScanThreads / 64];
  __shared__ int s_k, s_extent;
  const CompactBits w = {s_bits[0], s_bits[1], s_bits[2], s_bits[3]};
  const int tid = threadIdx.x, words = div_up(n_blocks, 32);
  int32_t* stack = free_list + kListHead;
  int32_t* marks = stack + n_blocks;
  for (int x0 = 0; x0 < n_blocks; x0 += kScanThreads) {
    const int x = x0 + tid;
    const uint64_t bits = __ballot(x < n_blocks && marks[min(x, n_blocks - 1)] == -1);
    if ((tid & 31) == 0 && x < n_blocks) {
      w.free[x >> 5] = (tid & 32) ? (uint32_t)(bits >> 32) : (uint32_t)bits;
      w.used[x >> 5] = 0;
    }
  }
  if (tid == 0) s_k = s_extent = 0;
  __syncthreads();
  const int all_entries = n_b * max_blocks;
  auto each_entry = [&](auto&& act) {      // four loads in flight
    for (int e0 = tid; e0 < all_entries; e0 += kScanThreads * 4) {
      int id[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = min(e0 + i * kScanThreads, all_entries - 1), b = e / max_blocks, j = e - b * max_blocks;
        const int entry = table[e];
        id[i] = e0 + i * kScanThreads < all_entries && j < entries_of(lens[b], max_blocks, shift) ? entry : -1;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((unsigned)id[i] < (unsigned)n_blocks) act(table + e0 + i * kScanThreads, id[i]);
    }
  };
  each_entry([&](int32_t*, int id) { atomicOr(&w.used[id >> 5], 1u << (id & 31)); });
  __syncthreads();
  uint32_t n_free, n_used;
  count_words(w, words, s_wave, [&](int i, uint32_t f) { return w.used[i] & ~f; }, n_free, n_used);
  __syncthreads();
  int k = largest_k<kScanThreads>(w, words, (int)n_used, tid);
  if (k) atomicMax(&s_k, k);
  __syncthreads();
  k = min(s_k, n_moves);
  for (int x0 = 0; x0 < n_blocks; x0 += kScanThreads) {
    const int x = x0 + tid;
    const uint64_t some = __ballot(x < n_blocks && settle(x, w, k, (int)n_free, (int)n_used, stack, marks, moves));
    if (some && (tid & 63) == 0) atomicMax(&s_extent, x + 64 - (int)__builtin_clzll(some));
  }
  for (int64_t i = 2 * (int64_t)k + tid; i < 2 * (int64_t)n_moves; i += kScanThreads) moves[i] = -1;
  if (tid == 0) free_list[0] = (int)n_free;
  __syncthreads();                         // (the workgroup's own stores to `moves` are read)
  if (k) each_entry([&](int32_t* entry, int id) {
    const int now = renamed(id, w, k, (int)n_used, moves);
    if (now != id) *entry = now;
  });
  if (tid == 0) *extent = s_extent;
}

// ---- copy ----------------------------------------------------------------------------------------
// Pages by pairs (from, to).  A workgroup takes kPieces 16-byte pieces of the keys, in the grid's second half of the values: of several
// pages where they are small (`group` of them), else part of one.  Loads go through the caches and stores past them: what several
// rows continue is read from memory once.  us for 7 copies of 1024 blocks of 64 KB / 2 of each of 33 x 65 of 128 KB / 2 x 16384 blocks moved,
// with what deals and frees them, on pages that no cache holds: 166 / 134 / 643; loads past the caches as well 217 / 140 / 627; keys and values
// of a page by one workgroup 188 / 137 / 666.  Repeated on the same pages: 168 / 107 / 642; stores through the caches 261 / 163; eight pieces a
// thread 165 / 113 / 675, two 169 / 106 / 652.
constexpr int kPerThread = 4, kPieces = kThreads * kPerThread;
__global__ __launch_bounds__(kThreads) void paged_copy_kernel(const int32_t* __restrict__ moves, int n_moves, unsigned char* __restrict__ K,
                                                              unsigned char* __restrict__ V, int32_t* __restrict__ deg, unsigned char* __restrict__ bounds,
                                                              int32_t* __restrict__ mass, int n_blocks, int page_pieces, int rows, int heads,
                                                              int bound_pieces, int group, int parts) {
  const bool values = blockIdx.x >= gridDim.x / 2;
  const int id = values ? blockIdx.x - gridDim.x / 2 : blockIdx.x;
  unsigned char* pool = values ? V : K;
  const int m0 = id / parts * group, part = id % parts, tid = threadIdx.x;
  const int n = min(group, n_moves - m0);
  auto pair = [&](int m, int& from, int& to) {
    from = moves[2 * m];
    to = moves[2 * m + 1];
    return (unsigned)from < (unsigned)n_blocks && (unsigned)to < (unsigned)n_blocks && from != to;
  };
  const int p0 = part * kPieces, total = parts > 1 ? min(kPieces, page_pieces - p0) : n * page_pieces;
  uint4 piece[kPerThread];
  int64_t at[kPerThread];
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int e = tid + i * kThreads;
    at[i] = -1;
    if (e < total) {
      const int m = parts > 1 ? 0 : e / page_pieces, p = parts > 1 ? p0 + e : e % page_pieces;
      int from, to;
      if (pair(m0 + m, from, to)) {
        at[i] = ((int64_t)to * page_pieces + p) * 16;
        const int64_t src = ((int64_t)from * page_pieces + p) * 16;
        piece[i] = *reinterpret_cast<const uint4*>(pool + src);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kPerThread; ++i)
    if (at[i] >= 0) stg16_stream(pool + at[i], piece[i]);
  if (values || part) return;
  for (int m = 0; m < n; ++m) {
    int from, to;
    if (!pair(m0 + m, from, to)) continue;
    if (deg)
      for (int i = tid; i < rows; i += kThreads) deg[(int64_t)to * rows + i] = deg[(int64_t)from * rows + i];
    if (bounds) {
      for (int i = tid; i < bound_pieces; i += kThreads)
        *reinterpret_cast<uint4*>(bounds + ((int64_t)to * bound_pieces + i) * 16) = *reinterpret_cast<const uint4*>(bounds + ((int64_t)from * bound_pieces + i) * 16);
      for (int i = tid; i < heads; i += kThreads) mass[(int64_t)to * heads + i] = mass[(int64_t)from * heads + i];
    }
  }
}

}  // namespace

hipError_t launch_paged_fork(int32_t* table, int32_t* lens, const int32_t* source, int32_t* free_list, int n_b, int max_blocks, int n_blocks,
                             int shift, int32_t* moves, int n_moves, int32_t* granted, hipStream_t st) {
  const bool counted = n_b > kRowsHere || n_b * max_blocks > kEntriesHere;
  if (counted) {
    ScopedTimer t("fork_count", st);
    hipLaunchKernelGGL(fork_count_kernel, dim3((unsigned)n_b), dim3(kThreads), 0, st, table, lens, source, n_b, max_blocks, n_blocks, shift, granted);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ScopedTimer t("fork_deal", st);
  // (One workgroup waits for no other: two rows, of which one continues the other, with their copy and trim 12.0 us against 12.6, both in
  // turn in one process, replayed by a graph 11.6 against 13.3; rows that follow each other in it cost 1 us each: eight 22.5 against 16.4.)
  const dim3 grid(n_b <= 2 ? 1u : (unsigned)(n_b < 256 ? n_b : 256));
  if (n_b <= kThreads)
    hipLaunchKernelGGL(fork_deal_kernel<1>, grid, dim3(kThreads), (size_t)n_b * 8, st, table, lens, source, free_list, n_b, max_blocks, n_blocks, shift,
                       moves, n_moves, granted, counted);
  else
    hipLaunchKernelGGL(fork_deal_kernel<16>, grid, dim3(kThreads), (size_t)n_b * 8, st, table, lens, source, free_list, n_b, max_blocks, n_blocks, shift,
                       moves, n_moves, granted, counted);
  return hipGetLastError();
}

size_t compact_scratch_bytes(int n_blocks) { return 64 + (32 + 4 * sizeof(uint32_t)) * (size_t)div_up(n_blocks, 32); }

hipError_t launch_paged_compact(int32_t* table, const int32_t* lens, int32_t* free_list, int n_b, int max_blocks, int n_blocks, int shift,
                                int32_t* moves, int n_moves, int32_t* extent, void* workspace, hipStream_t st) {
  const int words = div_up(n_blocks, 32);
  if (n_blocks <= kSmallBlocks && (int64_t)n_b * max_blocks <= kSmallEntries) {
    ScopedTimer t("compact_small", st);
    hipLaunchKernelGGL(compact_small_kernel, dim3(1), dim3(kScanThreads), 0, st, table, lens, free_list, n_b, max_blocks, n_blocks, shift, moves,
                       n_moves, extent);
    return hipGetLastError();
  }
  CompactScratch w;
  w.head = static_cast<int32_t*>(workspace);
  w.named = static_cast<uint8_t*>(workspace) + 64;
  w.bits.free = reinterpret_cast<uint32_t*>(w.named + (size_t)words * 32);
  w.bits.used = w.bits.free + words;
  w.bits.free_before = w.bits.used + words;
  w.bits.used_before = w.bits.free_before + words;
  const dim3 blocks((unsigned)div_up(n_blocks, kThreads)), threads(kThreads);
  const int across = div_up(max_blocks, kThreads * 4);
  const dim3 entries((unsigned)n_b, (unsigned)(across < 64 ? across : 64));
  hipError_t e;
#define CKV_STEP(name, kernel, grid, block, ...)                        \
  {                                                                     \
    ScopedTimer t(name, st);                                            \
    hipLaunchKernelGGL(kernel, grid, block, 0, st, __VA_ARGS__);        \
  }                                                                     \
  e = hipGetLastError();                                                \
  if (e != hipSuccess) return e
  CKV_STEP("compact_free", compact_free_kernel, blocks, threads, free_list, n_blocks, w, extent);
  CKV_STEP("compact_used", compact_used_kernel, entries, threads, table, lens, max_blocks, n_blocks, shift, w);
  CKV_STEP("compact_scan", compact_scan_kernel, dim3(1), dim3(kScanThreads), words, n_moves, w);
  CKV_STEP("compact_blocks", compact_blocks_kernel, blocks, threads, free_list, n_blocks, w, moves, n_moves, extent);
  CKV_STEP("compact_rename", compact_rename_kernel, entries, threads, table, lens, max_blocks, n_blocks, shift, w, moves);
#undef CKV_STEP
  return hipSuccess;
}

hipError_t launch_paged_copy(const int32_t* moves, int n_moves, void* K, void* V, int32_t* deg, void* bounds, int32_t* mass, int n_blocks, int heads,
                             int block_size, int row_bytes, hipStream_t st) {
  if (n_moves == 0) return hipSuccess;
  ScopedTimer t("paged_copy", st);
  const int pieces = heads * block_size * (row_bytes / 16);
  const int group = pieces < kPieces ? kPieces / pieces : 1, parts = div_up(pieces, kPieces);
  hipLaunchKernelGGL(paged_copy_kernel, dim3(2u * (unsigned)(div_up(n_moves, group) * parts)), dim3(kThreads), 0, st, moves, n_moves,
                     static_cast<unsigned char*>(K), static_cast<unsigned char*>(V), deg, static_cast<unsigned char*>(bounds), mass, n_blocks, pieces,
                     heads * block_size, heads, heads * 2 * (row_bytes / 16), group, parts);
  return hipGetLastError();
}

}  // namespace ckv
