// Attention of several new tokens of every sequence over a block-paged cache (Eq. 3 for each of them):
//   o_i = softmax_t(q_i . k_t * scale + ln N_t) V,   t up to the token's own position (or over the whole cache).
// The rows of one KV head's product are (new token, query head of the group) pairs, so that keys and values are read once for the
// group.  A workgroup takes 128 rows of one sequence and walks over its tokens in tiles of 64 (fp32: 32) that go from memory to LDS without
// passing registers, one tile ahead; a wave holds 32 rows: their queries, their running maximum and sum, and their sums of values.  Two
// workgroups share a CU, so that one's products run beside the other's softmax.
//
// The product is turned: S^T = K Q^T has a query row in each lane, so that the softmax of a row is a matter of one lane and its
// partner 32 lanes away, and what comes out of it is, without any exchange, the right operand of O^T += V^T P^T: the order in which
// the tokens of a matrix instruction are summed is free, and V is read from LDS in the order P has.
//   l += sum_t p_t,  O += sum_t p_t v_t,  p_t = 2^(c s_t - r),  c = scale log2 e;   where some c s_t > r + 8:  r' = max, l, O *= 2^(r - r')
// (a weight of 2^8 at most is as exact in bf16 and fp32 as one of 1, and most tiles rescale nothing).  ln N / scale is one more product of the
// chain that makes S: three bf16 parts of it by ones.
//
// What bounds it: many new tokens, the matrix cores and the exponentials beside them: a prompt of 16384 tokens (32 heads over 8, dim 128)
// 2070 us, 1062 TFLOP/s, where the library's product of 8192 cubed reaches 1370 to 1605 here (by the order of its right operand); four turns
// over 16384 970 to 985.  Few, memory: 16 requests of 1 to 8 tokens over 32768 298 us, 5.4 TB/s, what a copy reaches.
// Measured against an earlier step, whose figure is in brackets: 256 rows in eight waves, one workgroup a CU: 1068 TFLOP/s for the prompt
// (1070), 850 for the turns (885); 64 rows a wave: 740 to 794 (the sums no longer fit beside the rest); the next tile's S between this
// one's products with V 1010 to 1030; two halves of a workgroup in turn 1036; waves of their own for few rows 380 us (311).
#include <type_traits>

#include "ckv_internal.h"
#include "ckv_device.h"
#include "k4_attn.h"

namespace ckv {
namespace {

constexpr int kRows = 128;               // query rows of a workgroup
constexpr int kWaves = 4, kThreads = kWaves * 64;
constexpr float kWhole = -1.f;           // in the place of a first part's sum: the row's output has been written
constexpr float kNoPart = -2.f;          // in the place of a part's sum: there is no such part of this row, nothing else of it has been written
constexpr float kSlack = 8.f;            // how far (log2) a logit may exceed the reference before the sums are rescaled

constexpr int kValu = 0x2, kMfma = 0x8, kDsRead = 0x100;   // kinds of instructions, for the order that the compiler is asked for
typedef __attribute__((ext_vector_type(4))) short s16x4;

struct ChunkArgs {
  const unsigned char* q;
  int64_t q_row, q_head;                 // in bytes
  int n, n_b;
  const int32_t* starts;
  const unsigned char *K, *V;
  const int32_t* deg;
  PagedView paged;
  const int32_t* lens;
  int max_len, heads, g_shift;           // query heads per KV head = 1 << g_shift
  float c;                               // scale * log2 e
  int causal, slots, splits, span, tail;
  void* o;
  int o_dtype;
  float *o_part, *ml_part;               // [split][token][query head][dim] and [..][2], with more than one split;
};                                       // where only a tail is cut, [place from the end][KV head][split][row]..

// The rows of a place: tokens tok0 .. of sequence b.
struct Rows {
  int b, tok0, tokens, len, pos0, seen;  // pos0: position of the first of these tokens; seen: tokens that any of them sees
};

__device__ __forceinline__ bool rows_of(const ChunkArgs& a, int t_shift, int b, int part, int first, int last, int len, Rows& r) {
  r.b = b;
  r.tok0 = first + (part << t_shift);
  r.tokens = min(last - r.tok0, 1 << t_shift);
  if (part < 0 || r.tokens <= 0) return false;
  const int64_t cap = (int64_t)a.paged.max_blocks << a.paged.shift;
  r.len = (int)min((int64_t)min(max(len, 0), a.max_len), cap);
  r.pos0 = r.len - (last - r.tok0);
  r.seen = a.causal ? max(min(r.pos0 + r.tokens, r.len), 0) : r.len;
  return true;
}

// What a workgroup's waves tell each other of an order.
struct Order { int before[kWaves][64], used[kWaves]; };

// Which rows the workgroup at `slot` has, of a batch of up to 64: the longest sequence's first, so that those that start last are the shortest,
// and of a sequence the last ones, which see most.  A lane holds a sequence and counts the places before its own, a quarter of the
// sequences in each wave (all of them in every wave: 4.5 us more a workgroup beside another, with 64 sequences).  used: places that have rows.
// back: count from the end of those (`slot` becomes the place).  All threads of the workgroup take part.
__device__ __forceinline__ bool in_order(const ChunkArgs& a, int t_shift, int wave, int lane, bool back, Order& s, int& slot, int& used, Rows& r) {
  const int at = min(lane, a.n_b - 1), first = min(max(a.starts[at], 0), a.n), last = min(max(a.starts[at + 1], 0), a.n);
  const int count = lane < a.n_b ? (max(last - first, 0) + (1 << t_shift) - 1) >> t_shift : 0, len = a.lens[at];
  int before = 0;
  used = 0;
  for (int i = wave * (64 / kWaves); i < min((wave + 1) * (64 / kWaves), a.n_b); ++i) {
    const int l = __builtin_amdgcn_readlane(len, i), c = __builtin_amdgcn_readlane(count, i);
    if (l > len || (l == len && i < lane)) before += c;
    used += c;
  }
  s.before[wave][lane] = before;
  if (lane == 0) s.used[wave] = used;
  __syncthreads();
  before = used = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += s.before[w][lane];
    used += __builtin_amdgcn_readfirstlane(s.used[w]);
  }
  if (back) slot = used - 1 - slot;
  const uint64_t mine = __ballot(slot >= before && slot < before + count);
  if (!mine) return false;
  const int b = (int)__builtin_ctzll(mine), part = __builtin_amdgcn_readlane(before + count, b) - 1 - slot;
  return rows_of(a, t_shift, b, part, __builtin_amdgcn_readlane(first, b), __builtin_amdgcn_readlane(last, b), __builtin_amdgcn_readlane(len, b), r);
}

// These rows' tokens are cut into as many equal parts as spans of a.span tokens hold them.
__device__ __forceinline__ int parts_of(const ChunkArgs& a, int seen) { return max((int)(((int64_t)seen + a.span - 1) / a.span), 1); }

// What a tile of the cache looks like for each type.  PIECES: 16-byte pieces of a row; TILE: tokens.
template <typename T, int D>
struct Tile {
  static constexpr bool BF16 = std::is_same<T, __bf16>::value;
  static constexpr int RB = D * (int)sizeof(T), PIECES = RB / 16;
  static constexpr int SUB = BF16 ? 2 : 1;               // 32-token products of a tile
  static constexpr int TILE = 32 * SUB;
  static constexpr int BYTES = TILE * RB;
  static constexpr int ROWS_PER_LOAD = 64 / PIECES;      // of a wave
  static constexpr int LOADS = TILE / ROWS_PER_LOAD / kWaves;
  static_assert(LOADS * ROWS_PER_LOAD * kWaves == TILE, "whole loads per wave");
  // Which 16-byte slot of its row piece p sits in (an involution).  Keys: 16 rows, one piece of each, in different banks.  Values:
  // bf16, four rows of 64 bytes (a transposed read of half a wave); fp32, rows four apart, 128 bytes of each.
  __device__ static __forceinline__ int k_slot(int row, int p) { return p ^ (PIECES >= 16 ? row & 15 : (row >> 1) & 7); }
  __device__ static __forceinline__ int v_slot(int row, int p) {
    if constexpr (BF16) return p ^ ((PIECES == 16 ? row & 3 : (row >> 1) & 1) << 2);
    else return PIECES >= 16 ? p ^ (((row >> 2) & 1) << 3) : p;
  }
};

// 16 bytes a lane from memory into LDS, lane l's at lds + 16 l (lds: the same in all lanes).  As a builtin every later read of LDS
// would wait for it; here the wait is the one before the tile's barrier.  (The load has read m0 when it is issued; what the compiler had there is gone.)
__device__ __forceinline__ void to_lds16(const void* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "m0", "memory");
}
// the same from a base that all lanes share
__device__ __forceinline__ void to_lds16(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// x, as something that the compiler knows nothing of: what a rare path works out from it is not kept in registers for it
__device__ __forceinline__ int unknown(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// op over a lane and its partner 32 away
template <class Op>
__device__ __forceinline__ float with_partner(float x, Op&& op) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <typename T, int D, bool DEG>
__global__ __launch_bounds__(kThreads, 2) void chunk_attn_kernel(ChunkArgs a) {
  using L = Tile<T, D>;
  constexpr int SUB = L::SUB, DT = D / 32;
  extern __shared__ __attribute__((aligned(16))) unsigned char s_tiles[];     // two tiles of keys and values
  // A tile's ln N / scale: bf16, of each token the sum of three bf16 and zeros, a row of a product with ones; fp32, the number.
  __shared__ __attribute__((aligned(16))) typename std::conditional<L::BF16, uint4, float>::type s_bias[2][DEG ? L::TILE : 1];
  __shared__ uint64_t s_valid[2], s_odd;                 // a tile's tokens that count; those with a value that is no finite number
  __shared__ int s_seq;
  __shared__ Order s_order;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, col = lane & 31;

  // ---- which rows, which tokens: first every place's first part, then the others of the places that are cut
  const int kvh = blockIdx.x % a.heads, place = blockIdx.x / a.heads;
  const int t_shift = __builtin_ctz(kRows) - a.g_shift;  // tokens of a workgroup
  const int split = place < a.slots ? 0 : 1 + (place - a.slots) / a.tail;
  int used = a.slots, slot = split ? a.tail - 1 - (place - a.slots) % a.tail : place;
  Rows mine;
  if (a.n_b <= 64) {
    if (!in_order(a, t_shift, wave, lane, split > 0, s_order, slot, used, mine)) return;
  } else {
    // Sequence b has the places from (starts[b] >> t_shift) + min(starts[b], b) on.  With c tokens, c > 0, the first term grows by c >> t_shift at
    // least and the second by one: as many as it needs, or one more; one without tokens has none, or one.  Together no more than n tokens
    // of as many sequences need, whatever the number of those without any.  us for tables of 4 / 65 / 256 / 4096 rows, three of which have a
    // new token after 32768: 96 / 96 / 98 / 103 (a place for every row, which then fill the chip without parts: 94 / 226 / 631 / 923).
    if (split) slot = a.slots - 1 - slot;
    if (tid == 0) s_seq = 0;
    __syncthreads();
    int before = 0;
    for (int i = tid; i < a.n_b; i += kThreads) {
      const int s = min(max(a.starts[i], 0), a.n);
      before += (s >> t_shift) + min(s, i) <= slot;
    }
    if (before) atomicAdd(&s_seq, before);
    __syncthreads();
    const int b = s_seq - 1;
    if (b < 0) return;
    const int first = min(max(a.starts[b], 0), a.n), last = min(max(a.starts[b + 1], 0), a.n);
    if (!rows_of(a, t_shift, b, slot - (first >> t_shift) - min(first, b), first, last, a.lens[b], mine)) return;
  }
  const int b = mine.b, tok0 = mine.tok0, tokens = mine.tokens, len = mine.len, pos0 = mine.pos0, seen = mine.seen;
  const int rows = tokens << a.g_shift;
  const int row = wave * 32 + col;
  const bool live = row < rows;
  const int my_tok = min(row >> a.g_shift, tokens - 1), my_head = (kvh << a.g_shift) + (row & ((1 << a.g_shift) - 1));
  const int limit = a.causal ? pos0 + my_tok : len - 1;  // the last token that this row sees
  const int all_see = a.causal ? pos0 : len - 1;         // the last one that every row sees
  const int wave_last = a.causal ? pos0 + min((wave * 32 + 31) >> a.g_shift, tokens - 1) : len - 1;
  const bool idle = wave * 32 >= rows;

  // (no sequence is longer than kMostTokens: a few tiles behind the last one still have a number)
  const int from_end = used - 1 - slot;
  const int n_tiles = (seen + L::TILE - 1) / L::TILE, parts = from_end < a.tail ? parts_of(a, seen) : 1;
  const int tile0 = split < parts ? (int)((int64_t)n_tiles * split / parts) : 0, tile1 = split < parts ? (int)((int64_t)n_tiles * (split + 1) / parts) : 0;
  const int q_heads = a.heads << a.g_shift;
  const bool all_cut = a.tail == a.slots;
  const int64_t out_row = (int64_t)(tok0 + my_tok) * q_heads + my_head;
  const int64_t part_row = all_cut ? (int64_t)split * a.n * q_heads + out_row : (((int64_t)from_end * a.heads + kvh) * a.splits + split) * kRows + row;
  if (split >= parts) {                  // nothing: a weight of zero
    if (all_cut && live && half == 0) *reinterpret_cast<float2*>(&a.ml_part[2 * part_row]) = make_float2(-INFINITY, kNoPart);
    return;
  }
  const int32_t* table = a.paged.table + (int64_t)b * a.paged.max_blocks;
  const int shift = a.paged.shift, mask = (1 << shift) - 1;

  // ---- queries: lane (col, half) holds pieces 2 s + half of its row
  constexpr int QP = L::PIECES / 2;
  uint4 qf[QP];
  {
    const unsigned char* qr = a.q + (int64_t)(tok0 + my_tok) * a.q_row + (int64_t)my_head * a.q_head;
#pragma unroll
    for (int s = 0; s < QP; ++s) qf[s] = *reinterpret_cast<const uint4*>(qr + (2 * s + half) * 16);
  }

  // ---- where a lane reads in a tile: its keys' pieces (row col), and its values (bf16: of a 4 x 16 block that lanes 16 g ..
  // 16 g + 15 read transposed, tokens 4 half + .., channels 16 (g & 1) + ..; fp32: token 4 half, channel col).  The tile's other
  // rows are a constant away.
  using LdsAt = const __attribute__((address_space(3))) unsigned char*;
  const LdsAt lds_tiles = (LdsAt)s_tiles;
  int k_at[QP], v_at[DT];
#pragma unroll
  for (int st = 0; st < QP; ++st) k_at[st] = col * L::RB + L::k_slot(col, 2 * st + half) * 16;
#pragma unroll
  for (int d = 0; d < DT; ++d) {
    const int r = L::BF16 ? 4 * half + ((lane & 15) >> 2) : 4 * half;
    const int at = L::BF16 ? 64 * d + 32 * ((lane >> 4) & 1) + 8 * (lane & 3) : 128 * d + 4 * col;
    v_at[d] = L::BYTES + r * L::RB + L::v_slot(r, at >> 4) * 16 + (at & 15);
  }

  f32x16 acc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
  float ref = -INFINITY, sum = 0.f;

  // ---- staging: a load takes ROWS_PER_LOAD rows, wave w's loads one behind the other.  A lane holds the table's entry of one of the
  // tile's tokens, asked for a tile ahead.  Where a load's rows lie in one block, their place is a matter of scalars.
  constexpr int PER = L::ROWS_PER_LOAD, RB_SHIFT = __builtin_ctz(L::RB);
  const int r_lane = lane / L::PIECES, slot_in_row = lane % L::PIECES;
  const bool whole_loads = (1 << shift) >= PER;
  auto entry = [&](int t) { return table[min(t, seen - 1) >> shift]; };
  auto pool_row = [&](int e, int t) {                    // (an entry outside the pool: the pool's first rows, masked)
    return (unsigned)e < (unsigned)a.paged.n_blocks ? ((e * a.heads + kvh) << shift) + (t & mask) : 0;
  };
  int ent = 0;
  auto ask_entries = [&](int tile) { ent = entry(tile * L::TILE + (lane & (L::TILE - 1))); };
  const uint32_t lds0 = lds_address(s_tiles);
  int dg = 1;
  const float inv_c = 1.f / a.c;
  auto request = [&](int tile, int buf) __attribute__((always_inline)) {
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + (uint32_t)buf * 2 * L::BYTES + (uint32_t)wave * L::LOADS * 1024);
    const int first_row = __builtin_amdgcn_readfirstlane(wave * L::LOADS * PER);
    if (whole_loads) {
#pragma unroll
      for (int i = 0; i < L::LOADS; ++i) {
        const int r = first_row + i * PER;
        const uint64_t at = (uint64_t)(uint32_t)pool_row(__builtin_amdgcn_readlane(ent, r), tile * L::TILE + r) << RB_SHIFT;
        to_lds16(a.K + at, (uint32_t)(r_lane * L::RB + L::k_slot(r + r_lane, slot_in_row) * 16), to + i * 1024);
        to_lds16(a.V + at, (uint32_t)(r_lane * L::RB + L::v_slot(r + r_lane, slot_in_row) * 16), to + L::BYTES + i * 1024);
      }
    } else {
      const int l = unknown(lane);
      for (int i = 0; i < L::LOADS; ++i) {
        const int r = first_row + i * PER + l / L::PIECES;
        const uint64_t at = (uint64_t)(uint32_t)pool_row(__shfl(ent, r), tile * L::TILE + r) << RB_SHIFT;
        to_lds16(a.K + at + L::k_slot(r, l % L::PIECES) * 16, to + i * 1024);
        to_lds16(a.V + at + L::v_slot(r, l % L::PIECES) * 16, to + L::BYTES + i * 1024);
      }
    }
    if (DEG && wave == kWaves - 1) dg = a.deg[pool_row(ent, tile * L::TILE + (lane & (L::TILE - 1)))];
  };
  // what the last wave says of a tile's tokens: ln N / scale of each (the product's first addend), and which count
  auto describe = [&](int tile, int buf, int e) {
    if (wave == kWaves - 1) {
      const int i = lane & (L::TILE - 1);
      const bool ok = tile * L::TILE + i < seen && (unsigned)e < (unsigned)a.paged.n_blocks && dg > 0;
      if constexpr (DEG) {
        const float x = ok ? __log2f((float)dg) * inv_c : 0.f;
        if constexpr (L::BF16) {
          const __bf16 hi = (__bf16)x, mid = (__bf16)(x - (float)hi);
          const bf16x2 two = {hi, mid}, one = {(__bf16)(x - (float)hi - (float)mid), (__bf16)0.f};
          s_bias[buf][i] = make_uint4(__builtin_bit_cast(uint32_t, two), __builtin_bit_cast(uint32_t, one), 0, 0);
        } else if (lane < L::TILE) {
          s_bias[buf][i] = x;
        }
      }
      const uint64_t valid = __ballot(ok);
      if (lane == 0) s_valid[buf] = valid;
    }
  };

  if (tile0 < tile1) {
    ask_entries(tile0);
    request(tile0, 0);
    const int e0 = ent;
    ask_entries(tile0 + 1);
    describe(tile0, 0, e0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
#pragma unroll
  for (int s = 0; s < QP; ++s) asm volatile("" : "+v"(qf[s].x), "+v"(qf[s].y), "+v"(qf[s].z), "+v"(qf[s].w));
  for (int tile = tile0; tile < tile1; ++tile) {
    const int buf = (tile - tile0) & 1, t0 = tile * L::TILE;
    const bool more = tile + 1 < tile1;
    const int e_next = ent;
    if (more) {
      request(tile + 1, buf ^ 1);
      ask_entries(tile + 2);
    }
    const LdsAt tile_at = lds_tiles + buf * 2 * L::BYTES;
    const uint64_t valid = ((uint64_t)__builtin_amdgcn_readfirstlane((int)(s_valid[buf] >> 32)) << 32) |
                           (uint32_t)__builtin_amdgcn_readfirstlane((int)s_valid[buf]);
    const bool edge = t0 + L::TILE - 1 > all_see || valid != ~0ull;
    uint64_t odd = 0;
    if (edge) {
      // Some row must not see some token: a weight of zero is no mask where the value is no finite number.  Values of tokens
      // that do not count become zero; so do infinities and NaN, which are added to the rows that see them afterwards.
      if (tid == 0) s_odd = 0;
      __syncthreads();
      for (int p = unknown(tid); p < L::TILE * L::PIECES; p += kThreads) {
        const int r = p / L::PIECES;
        uint4* at = reinterpret_cast<uint4*>(s_tiles + (2 * buf + 1) * L::BYTES) + p;
        uint4 u = *at;
        uint32_t* w = reinterpret_cast<uint32_t*>(&u);
        bool changed = false, strange = false;
        if (!((valid >> r) & 1)) {
          u = make_uint4(0, 0, 0, 0);
          changed = true;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t keep = ~0u;
            if constexpr (L::BF16) {
              if ((w[i] & 0x7f80u) == 0x7f80u) keep &= 0xffff0000u;
              if ((w[i] & 0x7f800000u) == 0x7f800000u) keep &= 0x0000ffffu;
            } else {
              if ((w[i] & 0x7f800000u) == 0x7f800000u) keep = 0;
            }
            if (keep != ~0u) { w[i] &= keep; strange = true; }
          }
        }
        if (changed || strange) *at = u;
        if (strange) atomicOr(reinterpret_cast<unsigned long long*>(&s_odd), 1ull << r);
      }
      __syncthreads();
      odd = ((uint64_t)__builtin_amdgcn_readfirstlane((int)(s_odd >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)s_odd);
    }
    if (!idle && t0 <= wave_last) {
      // ---- S^T: lane (col, half), register i: token 8 (i / 4) + 4 half + i % 4 of its 32
      f32x16 s[SUB];
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[u][i] = 0.f;
      __builtin_amdgcn_s_setprio(1);       // (whoever has products to start goes first: 2172 -> 2136 us for a prompt of 16384)
#pragma unroll
      for (int st = 0; st < QP; ++st)
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
          const u32x4 kf = *(const __attribute__((address_space(3))) u32x4*)(tile_at + k_at[st] + u * 32 * L::RB);
          if constexpr (L::BF16) {
            s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[st]), s[u], 0, 0, 0);
          } else {
            const f32x4 kk = __builtin_bit_cast(f32x4, kf), qq = __builtin_bit_cast(f32x4, qf[st]);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[u] = __builtin_amdgcn_mfma_f32_32x32x2f32(kk[j], qq[j], s[u], 0, 0, 0);
          }
        }
      if constexpr (DEG) {               // one more product of each chain: ln N / scale by one
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
          if constexpr (L::BF16) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(&s_bias[buf][u * 32 + col]);
            const uint32_t o = half ? 0u : 0x3f80u;
            const u32x4 ones = {o | o << 16, o, 0u, 0u};
            s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, ones), s[u], 0, 0, 0);
          } else {
            s[u] = __builtin_amdgcn_mfma_f32_32x32x2f32(s_bias[buf][u * 32 + col], half ? 0.f : 1.f, s[u], 0, 0, 0);
          }
        }
      }
      if constexpr (L::BF16) {
        __builtin_amdgcn_sched_group_barrier(kDsRead, QP, 0);
#pragma unroll
        for (int i = 0; i < QP + (DEG ? SUB : 0); ++i) {
          __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
          __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kMfma, QP, 0);
      }
      __builtin_amdgcn_s_setprio(0);
      if (edge) {
        const int lim = unknown(limit - t0 - 4 * half);
        const uint64_t ok = valid >> (4 * half);
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int j = u * 32 + 8 * (i >> 2) + (i & 3);
            if (j > lim || !((ok >> j) & 1)) s[u][i] = -INFINITY;
          }
      }
      // ---- softmax against a reference that follows the maximum once it is 2^8 below it
      float top = s[0][0];
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
      top = with_partner(top, [](float x, float y) { return fmaxf(x, y); }) * a.c;
      if (__any(top > ref + kSlack)) {
        const float now = fmaxf(ref, top);
        const float f = now == -INFINITY ? 1.f : exp2_raw(ref - now);
        ref = now;
        sum *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[d][i] *= f;
      }
      const float base = ref == -INFINITY ? 0.f : ref;   // (a row that has seen nothing yet: all weights zero)
      if constexpr (L::BF16) {
        // Weights are rounded to bf16 for the product: 2^-8 of each at most, and their sum is taken of the rounded ones, so that they
        // still add up to one.  An output's error against 64 bits is 0.0021 of it (root of the mean square), 0.0016 by a bf16 output's own rounding.  The rest
        // of each as a second bf16 part, and a second product: a prompt of 16384 2095 -> 2913 us, four turns over 16384 1416 -> 1914, drafted
        // tokens over 32768 299 -> 321.
        const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            Piece p;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f32x2 w = {exp2_raw(fmaf(s[u][8 * k + 2 * i], a.c, -base)), exp2_raw(fmaf(s[u][8 * k + 2 * i + 1], a.c, -base))};
              p.p[i] = __builtin_convertvector(w, bf16x2);
              sum = __builtin_amdgcn_fdot2_f32_bf16(p.p[i], ones, sum, false);
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              union { s16x4 h[2]; bf16x8 v; } vt;
#pragma unroll
              for (int e = 0; e < 2; ++e)
                vt.h[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4*)(tile_at + v_at[d] + (u * 32 + 16 * k + 8 * e) * L::RB));
              acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt.v, p.v, acc[d], 0, 0, 0);
            }
          }
        __builtin_amdgcn_sched_group_barrier(kValu, 24, 1);
        __builtin_amdgcn_sched_group_barrier(kDsRead, 2 * DT, 1);
#pragma unroll
        for (int g = 0; g < 2 * SUB - 1; ++g)
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            __builtin_amdgcn_sched_group_barrier(kMfma, 1, 1);
            __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 1);
            __builtin_amdgcn_sched_group_barrier(kValu, 24 / DT, 1);
          }
        __builtin_amdgcn_sched_group_barrier(kMfma, DT, 1);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float w = exp2_raw(fmaf(s[0][i], a.c, -base));
          sum += w;
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            // (rows 8 i + 4 half + .. of a d have their slots alike)
            const float v = *(const __attribute__((address_space(3))) float*)(tile_at + v_at[d] + (8 * (i >> 2) + (i & 3)) * L::RB);
            acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, w, acc[d], 0, 0, 0);
          }
        }
      }
      // ---- values that are no finite numbers, as they are in the cache
      while (odd) {
        const int j = __builtin_ctzll(odd);
        odd &= odd - 1;
        const int t = t0 + j;
        const unsigned char* vr = a.V + ((uint64_t)(uint32_t)pool_row(entry(t), t) << RB_SHIFT);
        if (t <= limit) {
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int ch = 32 * d + 8 * (i >> 2) + 4 * half + (i & 3);
              float v;
              if constexpr (L::BF16) v = __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(vr)[ch] << 16);
              else v = reinterpret_cast<const float*>(vr)[ch];
              if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) acc[d][i] += v;
            }
        }
      }
    }
    if (more) describe(tile + 1, buf ^ 1, e_next);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  if (idle) return;
  sum = with_partner(sum, [](float x, float y) { return x + y; });
  if (!live) return;
  if (parts == 1) {
    if (all_cut && a.splits > 1 && half == 0) *reinterpret_cast<float2*>(&a.ml_part[2 * part_row]) = make_float2(0.f, kWhole);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const int64_t at = out_row * D + 32 * d + 8 * i4 + 4 * half;
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = sum == 0.f ? 0.f : acc[d][4 * i4 + i] * inv;
        if (a.o_dtype == CKV_BF16) {
          const f32x2 lo = {v[0], v[1]}, hi = {v[2], v[3]};
          const uint2 w = make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
                                     __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2)));
          *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.o) + at) = w;
        } else {
          *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.o) + at) = v;
        }
      }
    return;
  }
  if (half == 0) *reinterpret_cast<float2*>(&a.ml_part[2 * part_row]) = make_float2(ref, sum);
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = acc[d][4 * i4 + i];
      *reinterpret_cast<f32x4*>(&a.o_part[part_row * D + 32 * d + 8 * i4 + 4 * half]) = v;
    }
}

// The parts of a row put together, in the order of their numbers, by a wave: a lane takes D / 64 channels (D = 32: half of the lanes one
// each).  row: the first part's, the others `step` rows apart; to: the row of the output.  Only parts that do not exist are passed over: a weight
// of zero makes an infinite sum of values NaN, as it does in a row of one part.
template <int D>
__device__ __forceinline__ void merge_row(const float* __restrict__ o_part, const float* __restrict__ ml_part, int parts, int64_t row, int64_t step, int64_t to,
                                          int lane, void* __restrict__ o, int o_dtype) {
  constexpr int E = D == 128 ? 2 : 1;
  float m = -INFINITY, l = 0.f;
  if (lane < parts) {
    const float2 v = *reinterpret_cast<const float2*>(&ml_part[2 * (row + lane * step)]);
    m = v.x;
    l = v.y;
  }
  if (__builtin_amdgcn_readfirstlane(__float_as_uint(l)) == __float_as_uint(kWhole)) return;
  const float top = across_lanes<0x3f>(m, [](float x, float y) { return fmaxf(x, y); });
  const float w = m == -INFINITY ? 0.f : exp2f(m - top);
  const float den = across_lanes<0x3f>(w * l, [](float x, float y) { return x + y; });
  float x[E] = {};
  for (int s = 0; s < parts; ++s) {
    if (__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(l), s)) == kNoPart) continue;
    const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), s));
    const float* p = &o_part[(row + s * step) * D + E * (lane & (D / E - 1))];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = fmaf(p[e], f, x[e]);
  }
  if (E * lane >= D) return;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float r = over_sum(x[e], den);
    if (o_dtype == CKV_BF16) reinterpret_cast<uint16_t*>(o)[to * D + E * lane + e] = f32_to_bf16_rne(r);
    else reinterpret_cast<float*>(o)[to * D + E * lane + e] = r;
  }
}

// All rows, a wave each.
template <int D>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkArgs a, int64_t n_rows) {
  const int lane = threadIdx.x & 63, q_heads = a.heads << a.g_shift;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= n_rows) return;
  const int tok = (int)(row / q_heads);
  if (tok < a.starts[0] || tok >= min(a.starts[a.n_b], a.n)) return;
  merge_row<D>(a.o_part, a.ml_part, a.splits, row, n_rows, row, lane, a.o, a.o_dtype);
}

// The rows of the places that were cut: a workgroup takes kMergeRows of a place and a KV head.
constexpr int kMergeRows = 16;
template <int D>
__global__ __launch_bounds__(256) void chunk_merge_tail_kernel(ChunkArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t_shift = __builtin_ctz(kRows) - a.g_shift;
  const int group = blockIdx.x / (kRows / kMergeRows), row0 = blockIdx.x % (kRows / kMergeRows) * kMergeRows, kvh = group % a.heads;
  const int from_end = group / a.heads;
  __shared__ Order s_order;
  int slot = from_end, used;
  Rows w;
  if (!in_order(a, t_shift, wave, lane, true, s_order, slot, used, w)) return;
  const int parts = parts_of(a, w.seen);
  if (parts == 1) return;
  for (int r = row0 + wave; r < min(row0 + kMergeRows, w.tokens << a.g_shift); r += 4) {
    const int64_t to = (((int64_t)(w.tok0 + (r >> a.g_shift)) * a.heads + kvh) << a.g_shift) + (r & ((1 << a.g_shift) - 1));
    merge_row<D>(a.o_part, a.ml_part, parts, ((int64_t)group * a.splits) * kRows + r, kRows, to, lane, a.o, a.o_dtype);
  }
}

}  // namespace

namespace {
constexpr int kMostSplits = 64, kLeastSpan = 128, kSpan = 4096, kRounds = 3;
constexpr int kTailSplits = 4, kTailEighths = 4;
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }
int64_t most(int64_t a, int64_t b) { return a > b ? a : b; }
// the most parts that a call of up to max_len tokens is cut into
int64_t most_splits(int max_len) { return least(up(max_len, kLeastSpan), kMostSplits); }
int groups_at_once() { return 2 * cu_count(); }
int64_t tail_places(int heads) { return up(groups_at_once() * (int64_t)kTailEighths / 8, heads); }
}  // namespace

// How the tokens are cut.  Few places: so that every workgroup that fits on the chip has work, down to spans of kLeastSpan tokens; and down
// to kSpan tokens into kRounds times as many workgroups as fit, so that those that finish last are few.
// us with kRounds, kSpan = 3, 4096 / 3, 2048 / 6, 4096 / 10, 1024: 16 requests of 1 to 8 tokens over 32768 313 / 341 / 310 / 349; 39 single
// tokens and 1999 of another over 16384 922 / 930 / 953 / 1008.  33 tokens over 515 with kLeastSpan 128 / 256 / 512: 15.4 / 16.5 / 19.3.
// Places enough for kRounds rounds: the last half of a round (kTailEighths) in up to kTailSplits parts, of kSpan tokens or more (of 512 or more,
// 64 turns of 100 over 1000 took 176 us, not 154, and 8 of 1000 over 2000 274, not 252).  Four turns of 1024 to 2048 tokens over
// 16384 are three rounds and a little: 1537 us with whole places, 1434 so, 1428 with 8 parts, 1440 with a quarter of a round, 1446 with
// a whole one; a prompt of 16384 tokens stays as it is.  From one round on (kRounds 1): 39 single tokens beside 1999 975, not 908,
// 9 x 700 tokens over 1500 states 56, not 40.
ChunkCut chunk_cut(int n_b, int heads, int q_heads, int n, int max_len) {
  ChunkCut cut;
  cut.slots = n / (kRows / (q_heads / heads)) + (int)least(most(n, 1), n_b);   // (no more sequences than tokens have any)
  const int64_t groups = (int64_t)cut.slots * heads;
  if (groups >= (int64_t)kRounds * groups_at_once()) {
    cut.span = (int)(up(most(up(max_len, kTailSplits), kSpan), 64) * 64);
    cut.tail = n_b <= 64 && max_len > cut.span ? (int)least(tail_places(heads), cut.slots - 1) : 0;
    cut.splits = cut.tail ? (int)up(max_len, cut.span) : 1;
    return cut;
  }
  const int64_t fill = least(up(groups_at_once(), groups), up(max_len, kLeastSpan));
  const int64_t even = least(up((int64_t)kRounds * groups_at_once(), groups), up(max_len, kSpan));
  const int64_t splits = least(most(fill, even), kMostSplits);
  cut.span = (int)(up(up(max_len, splits), 64) * 64);
  cut.splits = (int)up(max_len, cut.span);
  cut.tail = cut.slots;
  return cut;
}

// (max, sum) pairs, up to the next 16 bytes, then the sums of values
static size_t part_bytes(int64_t parts, int dim) { return (size_t)(parts * 8 + 15) / 16 * 16 + (size_t)parts * dim * 4; }
static int64_t part_rows(const ChunkCut& cut, int heads, int64_t rows) {
  return cut.splits <= 1 ? 0 : cut.splits * (cut.tail == cut.slots ? rows : (int64_t)cut.tail * heads * kRows);
}

size_t chunk_workspace_bytes(const ChunkCut& cut, int heads, int64_t rows, int dim) { return part_bytes(part_rows(cut, heads, rows), dim); }

// All places are cut where there are fewer than kRounds * groups_at_once() of them, of kRows rows at most, into as many parts more as make
// up the difference; and none into more than most_splits().  A tail is cut where a batch of up to 64 can have as many places.
size_t chunk_reserve_bytes(int heads, int q_heads, int n, int max_len, int dim) {
  const int64_t some = most_splits(max_len), full = (int64_t)kRows * kRounds * groups_at_once(), rows = (int64_t)n * q_heads;
  if (some <= 1) return 0;
  const bool tail = ((int64_t)n / (kRows / (q_heads / heads)) + (n < 64 ? n : 64)) * heads >= (int64_t)kRounds * groups_at_once();
  return part_bytes(most(least(rows * some, full + least(rows, full)), tail ? tail_places(heads) * heads * kRows * kTailSplits : 0), dim);
}

hipError_t launch_chunk_attn(const ChunkCall& c, int dtype, int dim, hipStream_t st) {
  const ChunkCut cut = chunk_cut(c.n_b, c.heads, c.q_heads, c.n, c.max_len);
  ChunkArgs a{};
  a.q = static_cast<const unsigned char*>(c.q);
  a.q_row = c.q_row; a.q_head = c.q_head;
  a.n = c.n; a.n_b = c.n_b; a.starts = c.starts;
  a.K = static_cast<const unsigned char*>(c.K); a.V = static_cast<const unsigned char*>(c.V); a.deg = c.deg;
  a.paged = c.paged; a.lens = c.lens; a.max_len = c.max_len; a.heads = c.heads;
  a.g_shift = __builtin_ctz(c.q_heads / c.heads);
  a.c = c.scale * kLog2e;
  a.causal = c.causal; a.slots = cut.slots; a.splits = cut.splits; a.span = cut.span; a.tail = cut.tail;
  a.o = c.o; a.o_dtype = c.o_dtype;
  const int64_t rows = (int64_t)c.n * c.q_heads;
  a.ml_part = static_cast<float*>(c.workspace);
  a.o_part = a.ml_part + (part_rows(cut, c.heads, rows) * 2 + 3) / 4 * 4;
  const dim3 grid((unsigned)((cut.slots + (int64_t)cut.tail * (cut.splits - 1)) * c.heads));
  hipError_t e = hipErrorInvalidValue;
#define CKV_CHUNK_DEG(T, D, DEG)                                                                                             \
  do {                                                                                                                \
    static KernelSetup setup;                                                                                         \
    constexpr size_t lds = 4 * Tile<T, D>::BYTES;                                                                     \
    e = kernel_setup(reinterpret_cast<const void*>(&chunk_attn_kernel<T, D, DEG>), lds, setup);                         \
    if (e != hipSuccess) return e;                                                                                    \
    {                                                                                                                 \
      ScopedTimer t("chunk_attn", st);                                                                                \
      hipLaunchKernelGGL((chunk_attn_kernel<T, D, DEG>), grid, dim3(kThreads), lds, st, a);                           \
    }                                                                                                                 \
    e = hipGetLastError();                                                                                            \
    if (e == hipSuccess && cut.splits > 1) {                                                                          \
      ScopedTimer t("chunk_merge", st);                                                                               \
      if (cut.tail == cut.slots)                                                                                      \
        hipLaunchKernelGGL((chunk_merge_kernel<D>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, a, rows);     \
      else                                                                                                            \
        hipLaunchKernelGGL((chunk_merge_tail_kernel<D>), dim3((unsigned)(cut.tail * c.heads * (kRows / kMergeRows))), dim3(256), 0, st, a); \
      e = hipGetLastError();                                                                                          \
    }                                                                                                                 \
  } while (0)
#define CKV_CHUNK(T, D)                    \
  do {                                     \
    if (c.deg) CKV_CHUNK_DEG(T, D, true);  \
    else CKV_CHUNK_DEG(T, D, false);       \
  } while (0)
  if (dtype == CKV_BF16) {
    if (dim == 64) CKV_CHUNK(__bf16, 64);
    else if (dim == 128) CKV_CHUNK(__bf16, 128);
  } else {
    if (dim == 32) CKV_CHUNK(float, 32);
    else if (dim == 64) CKV_CHUNK(float, 64);
    else if (dim == 128) CKV_CHUNK(float, 128);
  }
#undef CKV_CHUNK
#undef CKV_CHUNK_DEG
  return e;
}

}  // namespace ckv
