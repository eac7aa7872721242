// Block tables and slot maps of a block-paged cache, built on the GPU: which blocks a step's new tokens go to, the blocks that
// sequences give back, and the copy of ragged rows into their slots.
//
// Free list: int32 [4 + 2 n_blocks].  Word 0: the number c of free blocks, word 1: an arrival counter that is zero between
// calls, words 2 and 3 unused; then the stack, whose first c entries are the free blocks, the next one to be dealt last; then one
// mark a block, -1 for a free one and INT_MAX for one that is dealt (a block that is given back twice is taken once).
#include "ckv_internal.h"
#include "ckv_device.h"

namespace ckv {
namespace {

constexpr int kListHead = 4;
constexpr int kInUse = INT32_MAX;

__device__ __forceinline__ int blocks_of(int tokens, int shift) { return (tokens >> shift) + ((tokens & ((1 << shift) - 1)) != 0); }

// Sums over this thread and the threads before it, each cut to `most` (x is, and 2 * most fits 32 bits); `all` receives the
// sum of the whole workgroup.  s_wave: one word a wave.
template <int THREADS>
__device__ __forceinline__ uint32_t scan_capped(uint32_t x, uint32_t most, uint32_t* s_wave, uint32_t& all) {
  constexpr int W = THREADS / 64;
#define CKV_SCAN_STEP(ctrl, rows) x = min(x + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xF, false), most)
  CKV_SCAN_STEP(0x111, 0xF);               // a row of 16: one, two, four, eight lanes up
  CKV_SCAN_STEP(0x112, 0xF);
  CKV_SCAN_STEP(0x114, 0xF);
  CKV_SCAN_STEP(0x118, 0xF);
  CKV_SCAN_STEP(0x142, 0xA);               // the last lane of rows 0 and 2 into rows 1 and 3
  CKV_SCAN_STEP(0x143, 0xC);               // lane 31 into rows 2 and 3
#undef CKV_SCAN_STEP
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 63) s_wave[wave] = x;
  __syncthreads();
  uint32_t before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    if (w == wave) before = all;
    all = min(all + s_wave[w], most);
  }
  __syncthreads();                         // (s_wave is free again)
  return min(x + before, most);
}

// at[e] = first i in [0, n) with end[i] > x[e], n - 1 where there is none (end does not fall): the searches' reads of LDS go together
template <int E>
__device__ __forceinline__ void owners_of(const int32_t* end, int n, const int (&x)[E], int (&at)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) at[e] = 0;
  for (int step = 1 << (31 - __clz(n)); step > 0; step >>= 1) {
    int v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = end[min(at[e] + step, n) - 1];
#pragma unroll
    for (int e = 0; e < E; ++e) at[e] += at[e] + step <= n && v[e] <= x[e] ? step : 0;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) at[e] = min(at[e], n - 1);
}

constexpr int kReserveThreads = 256;

// Every workgroup works out for itself who gets what (two running sums over the requests, in LDS), then writes its share of
// the slots and of the table entries: a request's j-th new token is token L + j of its row, in the entry the row has there
// already or in one that this call deals, the i-th block dealt being the i-th from the stack's top.  Nothing that one workgroup
// writes is read by another: lengths and the number of free blocks change when the last one has read them.
//
// What bounds it: a chain of trips to memory (lengths; entry or stack; store) and of reads of LDS, for 64 requests of one token
// each the whole of its 4.3 us.  So a thread takes ROWS requests in a row and searches for the owners of its SLOTS slots
// together (1000 requests, 256 at a time, slot by slot: 12.1 us, now 7.0; 33 prompts of 135000 slots 8.8, now 7.9).
// dynamic LDS: 12 bytes a request
template <int ROWS, int SLOTS>   // a thread's requests and slots
__global__ __launch_bounds__(kReserveThreads) void paged_reserve_kernel(
    int32_t* __restrict__ table, int32_t* __restrict__ lens, const int32_t* __restrict__ n_new, int32_t* __restrict__ free_list,
    int n_b, int max_blocks, int n_blocks, int shift, int32_t* __restrict__ slots, int n_slots, int32_t* __restrict__ starts,
    int32_t* __restrict__ granted) {
  extern __shared__ int32_t s_dyn[];
  int32_t *s_end = s_dyn, *s_dealt = s_dyn + n_b, *s_len = s_dyn + 2 * n_b;   // sums up to each request; its length, -1: refused
  __shared__ uint32_t s_wave[kReserveThreads / 64];
  __shared__ int s_last;
  const int tid = threadIdx.x, b0 = tid * ROWS;
  int len[ROWS], fresh[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    len[r] = lens[min(b0 + r, n_b - 1)];
    fresh[r] = n_new[min(b0 + r, n_b - 1)];
  }
  const int n_free = min(max(free_list[0], 0), n_blocks);
  const int32_t* stack = free_list + kListHead;
  int32_t* marks = free_list + kListHead + n_blocks;
  const int64_t row_tokens = (int64_t)max_blocks << shift;
  const uint32_t most_tokens = (uint32_t)n_slots + 1, most_blocks = (uint32_t)n_blocks + 1;   // (more than there is: how much more does not matter)
  // x[r] := sums over the requests up to each, cut to `most`
  auto sums = [&](uint32_t (&x)[ROWS], uint32_t most) {
#pragma unroll
    for (int r = 1; r < ROWS; ++r) x[r] = min(x[r] + x[r - 1], most);
    uint32_t all;
    const uint32_t upto = scan_capped<kReserveThreads>(x[ROWS - 1], most, s_wave, all);
    // (what is before this thread: the scan of the thread before, as cut sums cannot be taken apart)
    uint32_t before = (uint32_t)__shfl_up((int)upto, 1);
    if ((tid & 63) == 63) s_wave[tid >> 6] = upto;
    __syncthreads();
    if ((tid & 63) == 0) before = tid ? s_wave[(tid >> 6) - 1] : 0u;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROWS; ++r) x[r] = min(x[r] + before, most);
  };
  uint32_t end[ROWS], dealt[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    fresh[r] = b0 + r < n_b ? max(fresh[r], 0) : 0;
    end[r] = min((uint32_t)fresh[r], most_tokens);
  }
  sums(end, most_tokens);
  bool fits[ROWS], needs[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    fits[r] = b0 + r < n_b && len[r] >= 0 && (int64_t)len[r] + fresh[r] <= row_tokens && end[r] <= (uint32_t)n_slots;
    const int need = fits[r] ? blocks_of(len[r] + fresh[r], shift) - blocks_of(len[r], shift) : 0;
    needs[r] = need > 0;
    dealt[r] = min((uint32_t)need, most_blocks);
  }
  sums(dealt, most_blocks);
  uint32_t dealt_here = 0;                 // up to the last request here that is served and needs any
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const bool ok = fits[r] && (!needs[r] || dealt[r] <= (uint32_t)n_free);
    if (b0 + r < n_b) {
      s_end[b0 + r] = (int)min(end[r], (uint32_t)n_slots);
      s_dealt[b0 + r] = (int)dealt[r];
      s_len[b0 + r] = ok ? len[r] : -1;
      if (ok && needs[r]) dealt_here = dealt[r];
    }
  }
  for (int w = 1; w < 64; w *= 2) dealt_here = max(dealt_here, (uint32_t)__shfl_xor((int)dealt_here, w));
  if ((tid & 63) == 0) s_wave[tid >> 6] = dealt_here;
  __syncthreads();
  uint32_t take_all = 0;
#pragma unroll
  for (int w = 0; w < kReserveThreads / 64; ++w) take_all = max(take_all, s_wave[w]);
  const int total = s_end[n_b - 1], take = (int)take_all, first = blockIdx.x * kReserveThreads * SLOTS;
  const bool deals = first < take;         // (no request takes more blocks than tokens: block i goes with slot i)
  int slot[SLOTS], owner[SLOTS], taker[SLOTS];
#pragma unroll
  for (int e = 0; e < SLOTS; ++e) slot[e] = first + e * kReserveThreads + tid;
  owners_of(s_end, n_b, slot, owner);
  if (deals) owners_of(s_dealt, n_b, slot, taker);
  int off[SLOTS], blk[SLOTS], fresh_blk[SLOTS];                // a slot's offset in its block, -1: none
  const int32_t* from[SLOTS];
#pragma unroll
  for (int e = 0; e < SLOTS; ++e) {
    const int b = owner[e], had = s_len[b];
    const int start = b ? s_end[b - 1] : 0, before = b ? s_dealt[b - 1] : 0;
    off[e] = -1;
    from[e] = stack;
    if (slot[e] < total && had >= 0) {
      const int t = had + (slot[e] - start), have = blocks_of(had, shift), at = t >> shift;
      off[e] = t & ((1 << shift) - 1);
      from[e] = at < have ? table + (int64_t)b * max_blocks + at : stack + max(n_free - 1 - (before + (at - have)), 0);
    }
  }
#pragma unroll
  for (int e = 0; e < SLOTS; ++e) {
    blk[e] = *from[e];
    if (deals) fresh_blk[e] = stack[max(n_free - 1 - min(slot[e], take), 0)];
  }
#pragma unroll
  for (int e = 0; e < SLOTS; ++e)
    if (slot[e] < n_slots) slots[slot[e]] = off[e] >= 0 && (unsigned)blk[e] < (unsigned)n_blocks ? (blk[e] << shift) + off[e] : -1;
  if (deals) {
#pragma unroll
    for (int e = 0; e < SLOTS; ++e) {
      const int b = taker[e], k = slot[e] - (b ? s_dealt[b - 1] : 0);
      if (slot[e] < take) {
        table[(int64_t)b * max_blocks + blocks_of(s_len[b], shift) + k] = fresh_blk[e];
        if ((unsigned)fresh_blk[e] < (unsigned)n_blocks) marks[fresh_blk[e]] = kInUse;
      }
    }
  }
  if (blockIdx.x == 0) {
    for (int b = tid; b < n_b; b += kReserveThreads) {
      if (starts) starts[b + 1] = s_end[b];
      if (granted) granted[b] = s_len[b] >= 0;
    }
    if (starts && tid == 0) starts[0] = 0;
  }
  if (gridDim.x > 1) {
    __syncthreads();                       // (what this workgroup read has arrived: it has been stored or compared)
    if (tid == 0) s_last = atomicAdd(&free_list[1], 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!s_last) return;
  } else {
    __syncthreads();
  }
  for (int b = tid; b < n_b; b += kReserveThreads)
    if (s_len[b] >= 0) lens[b] = s_len[b] + (s_end[b] - (b ? s_end[b - 1] : 0));   // (a request that is served has all of its slots)
  if (tid == 0) {
    free_list[0] = n_free - take;
    if (gridDim.x > 1) atomicExch(&free_list[1], 0);
  }
}

constexpr int kReturnThreads = 1024;

// Blocks back onto the stack, in one workgroup: the order on the stack is that of the entries, the last one first, so that a
// reservation that is taken back leaves the stack as it was.  An entry outside the pool, or one whose block is free already,
// is passed over; of several entries with the same block one is taken: each leaves its place in the block's mark, and the
// least one stays.  Whoever finds another place there (or a free block) says so, and only then are the marks read again.
// TABLE: the entries of each row behind new_lens[b] tokens, which become -1; else the n_ids entries of `entries`.
// A thread takes kPer entries at a time, neighbours neighbouring ones, and asks for them together; the entries before its own
// are counted by ballots, one word for 64 of them.  Bound by its trips to memory (lengths, entries, marks, stores: 4.7 us for 64 rows
// that give back four blocks) and, for thousands of entries, by one CU's scattered ones (33 rows of 4200 entries 19 us).
// With four entries in a row a thread and their rows sought one after the other 7.4 and 21.
// dynamic LDS (TABLE): 8 bytes a row
constexpr int kPer = 64 / (kReturnThreads / 64);
template <bool TABLE>
__global__ __launch_bounds__(kReturnThreads) void paged_return_kernel(int32_t* __restrict__ entries, int n_ids, int max_blocks,
                                                                      int n_b, int32_t* __restrict__ lens,
                                                                      const int32_t* __restrict__ new_lens,
                                                                      int32_t* __restrict__ free_list, int n_blocks, int shift) {
  extern __shared__ int32_t s_end[];       // entries up to each row, the last row first
  int32_t* s_last = s_end + n_b;           // and the end of its entries
  __shared__ uint32_t s_wave[kReturnThreads / 64];
  __shared__ int s_again, s_count[64], s_total;
  const int tid = threadIdx.x;
  int32_t* stack = free_list + kListHead;
  int32_t* marks = free_list + kListHead + n_blocks;
  int n_free = min(max(free_list[0], 0), n_blocks);
  int total = n_ids;
  if (tid == 0) s_again = 0;
  if (TABLE) {
    uint32_t sum = 0;
    for (int r0 = 0; r0 < n_b; r0 += kReturnThreads) {
      const int r = r0 + tid, b = n_b - 1 - r;
      uint32_t count = 0;
      int last = 0;
      if (r < n_b) {
        const int len = lens[b], cut = new_lens[b];
        last = min(blocks_of(len, shift), max_blocks);
        if (cut >= 0 && cut < len) {
          count = (uint32_t)max(last - blocks_of(cut, shift), 0);
          lens[b] = cut;                   // (this thread alone reads it)
        }
      }
      uint32_t all;
      const uint32_t end = scan_capped<kReturnThreads>(count, 0x7fffffffu, s_wave, all) + sum;
      if (r < n_b) { s_end[r] = (int)end; s_last[r] = last; }
      sum += all;
    }
    total = (int)sum;
  }
  __syncthreads();
  const int lane = tid & 63, wave = tid >> 6;
  for (int p0 = 0; p0 < total; p0 += kReturnThreads * kPer) {
    int p[kPer], row[kPer], id[kPer], found[kPer];
    int64_t at[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) p[e] = p0 + e * kReturnThreads + tid;
    if (TABLE) owners_of(s_end, n_b, p, row);
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      at[e] = -1;
      if (p[e] < total) {
        if (TABLE) at[e] = (int64_t)(n_b - 1 - row[e]) * max_blocks + s_last[row[e]] - 1 - (p[e] - (row[e] ? s_end[row[e] - 1] : 0));
        else at[e] = n_ids - 1 - p[e];
      }
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) id[e] = at[e] >= 0 ? entries[at[e]] : -1;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      if ((unsigned)id[e] >= (unsigned)n_blocks) id[e] = -1;
      found[e] = id[e] >= 0 ? atomicMin(&marks[id[e]], p[e]) : kInUse;
      if (TABLE && at[e] >= 0) entries[at[e]] = -1;
    }
    bool again = false;
#pragma unroll
    for (int e = 0; e < kPer; ++e) again |= found[e] != kInUse;
    if (again) s_again = 1;
    __syncthreads();                       // (every mark has been lowered: its old value is here)
    if (s_again) {
#pragma unroll
      for (int e = 0; e < kPer; ++e)
        if (id[e] >= 0 && __hip_atomic_load(&marks[id[e]], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != p[e]) id[e] = -1;
    }
    uint64_t taken[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      taken[e] = __ballot(id[e] >= 0);
      if (lane == 0) s_count[e * (kReturnThreads / 64) + wave] = (int)__popcll(taken[e]);
    }
    __syncthreads();                       // (and all marks have been read)
    if (wave == 0) {
      const int upto = (int)wave_inclusive_scan((uint32_t)s_count[lane]);
      s_count[lane] = upto - s_count[lane];
      if (lane == 63) s_total = upto;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (id[e] >= 0) {
        const int to = n_free + s_count[e * (kReturnThreads / 64) + wave] + (int)__popcll(taken[e] & ((1ull << lane) - 1));
        if (to < n_blocks) stack[to] = id[e];
        __hip_atomic_store(&marks[id[e]], -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    n_free = min(n_free + s_total, n_blocks);
    if (p0 + kReturnThreads * kPer < total) {
      if (tid == 0) s_again = 0;
      __builtin_amdgcn_s_waitcnt(0);       // (the next ones may hold the same blocks)
      __syncthreads();
    }
  }
  if (tid == 0) free_list[0] = n_free;
}

// Rows of k and v [n, heads, dim] into the pool by their slots (block * block_size + offset), degree 1; a slot outside the
// pool is passed over.  A thread takes 16-byte pieces of both tensors, consecutive threads consecutive ones of a row, and asks for
// eight before it stores one.  Bound by its bytes: 50021 rows of 8 heads of 128 bf16, 411 MB read and written, take 80 us on inputs
// that are new each time, 5.2 TB/s, as much as torch's copy of 1 GiB (this library's row copy of 8 GiB 6.3).  Stores that keep the
// pages in the caches 84; the same inputs over and over, half of them still there, 64.
constexpr int kWriteThreads = 256, kWritePieces = 4;
__global__ __launch_bounds__(kWriteThreads) void paged_write_kernel(
    const unsigned char* __restrict__ k, const unsigned char* __restrict__ v, RowStrides ks, RowStrides vs, const int32_t* __restrict__ slots, int n,
    unsigned char* __restrict__ K_pool, unsigned char* __restrict__ V_pool, int32_t* __restrict__ deg_pool, int heads, int pieces_per_row, int shift, int n_blocks, int rows_per_group) {
  const int per_row = heads * pieces_per_row;
  const int r0 = blockIdx.x * rows_per_group, r1 = min(r0 + rows_per_group, n), total = (r1 - r0) * per_row;
  for (int e0 = threadIdx.x; e0 < total; e0 += kWriteThreads * kWritePieces) {
    uint4 a[kWritePieces], c[kWritePieces];
    int slot[kWritePieces], h[kWritePieces], piece[kWritePieces];
#pragma unroll
    for (int u = 0; u < kWritePieces; ++u) {
      const int e = min(e0 + u * kWriteThreads, total - 1);
      const int r = r0 + e / per_row, x = e % per_row;
      h[u] = x / pieces_per_row;
      piece[u] = x % pieces_per_row;
      slot[u] = slots[r];
      a[u] = ldg16_stream(k + (r * ks.row + h[u] * ks.head + piece[u] * 16));
      c[u] = ldg16_stream(v + (r * vs.row + h[u] * vs.head + piece[u] * 16));
    }
#pragma unroll
    for (int u = 0; u < kWritePieces; ++u) {
      if (e0 + u * kWriteThreads >= total || slot[u] < 0 || (slot[u] >> shift) >= n_blocks) continue;
      const int64_t row = ((((int64_t)(slot[u] >> shift) * heads + h[u]) << shift) + (slot[u] & ((1 << shift) - 1)));
      stg16_stream(K_pool + (row * pieces_per_row + piece[u]) * 16, a[u]);
      stg16_stream(V_pool + (row * pieces_per_row + piece[u]) * 16, c[u]);
      if (piece[u] == 0 && deg_pool) deg_pool[row] = 1;
    }
  }
}

}  // namespace

hipError_t launch_paged_reserve(int32_t* table, int32_t* lens, const int32_t* n_new, int32_t* free_list, int n_b, int max_blocks,
                                int n_blocks, int shift, int32_t* slots, int n_slots, int32_t* starts, int32_t* granted,
                                hipStream_t st) {
  ScopedTimer t("paged_reserve", st);
  // A workgroup more is one more to count itself in, a slot more of a thread lengthens its chain.  us with one / four / eight slots a
  // thread, 33 requests: 1000 slots 4.8 / 6.2 / 8.2, 8192 5.6 / 7.1 / 9.4, 32768 6.0 / 8.0 / 10.2, 65536 7.3 / 8.0 / 10.8, 135168 10.4 /
  // 8.2 / 10.7, 524288 28.1 / 12.5 / 12.2; 1000 requests: 4000 7.0 / 10.2 / 13.3, 65536 8.8 / 10.3 / 13.8.  (The border could be higher.)
  const bool few = n_slots <= 32 * kReserveThreads;
  const int groups = n_slots > 0 ? div_up(n_slots, kReserveThreads * (few ? 1 : 4)) : 1;
#define CKV_RESERVE(rows, slots_each)                                                                                      \
  hipLaunchKernelGGL((paged_reserve_kernel<rows, slots_each>), dim3((unsigned)groups), dim3(kReserveThreads), (size_t)n_b * 12, st, table, \
                     lens, n_new, free_list, n_b, max_blocks, n_blocks, shift, slots, n_slots, starts, granted)
#define CKV_RESERVE_ROWS(slots_each)                                 \
  do {                                                               \
    if (n_b <= kReserveThreads) CKV_RESERVE(1, slots_each);          \
    else if (n_b <= 4 * kReserveThreads) CKV_RESERVE(4, slots_each); \
    else CKV_RESERVE(16, slots_each);                                \
  } while (0)
  if (few) CKV_RESERVE_ROWS(1);
  else CKV_RESERVE_ROWS(4);
#undef CKV_RESERVE_ROWS
#undef CKV_RESERVE
  return hipGetLastError();
}

hipError_t launch_paged_trim(int32_t* table, int32_t* lens, const int32_t* new_lens, int32_t* free_list, int n_b, int max_blocks,
                             int n_blocks, int shift, hipStream_t st) {
  ScopedTimer t("paged_trim", st);
  hipLaunchKernelGGL((paged_return_kernel<true>), dim3(1), dim3(kReturnThreads), (size_t)n_b * 8, st, table, 0, max_blocks, n_b,
                     lens, new_lens, free_list, n_blocks, shift);
  return hipGetLastError();
}

hipError_t launch_paged_free(const int32_t* ids, int n, int32_t* free_list, int n_blocks, hipStream_t st) {
  if (n == 0) return hipSuccess;
  ScopedTimer t("paged_free", st);
  hipLaunchKernelGGL((paged_return_kernel<false>), dim3(1), dim3(kReturnThreads), 0, st, const_cast<int32_t*>(ids), n, 0, 0,
                     static_cast<int32_t*>(nullptr), static_cast<const int32_t*>(nullptr), free_list, n_blocks, 0);
  return hipGetLastError();
}

hipError_t launch_paged_write(const void* k, RowStrides ks, const void* v, RowStrides vs, const int32_t* slots, int n, void* K_pool, void* V_pool,
                              int32_t* deg_pool, int heads, int row_bytes, int shift, int n_blocks,
                              hipStream_t st) {
  if (n == 0) return hipSuccess;
  ScopedTimer t("paged_write", st);
  const int per_row = heads * (row_bytes / 16), most = kWriteThreads * kWritePieces;
  const int rows = per_row < most ? most / per_row : 1;
  hipLaunchKernelGGL(paged_write_kernel, dim3((unsigned)div_up(n, rows)), dim3(kWriteThreads), 0, st,
                     static_cast<const unsigned char*>(k), static_cast<const unsigned char*>(v), ks, vs, slots, n,
                     static_cast<unsigned char*>(K_pool), static_cast<unsigned char*>(V_pool), deg_pool, heads, row_bytes / 16, shift,
                     n_blocks, rows);
  return hipGetLastError();
}

}  // namespace ckv
