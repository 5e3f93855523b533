// Attention of packed query rows over a paged grouped-query KV cache, on the matrix cores: the body of a
// workgroup, shared by the launch of its own (rows_attn.hip) and the one that it shares with the sweep
// (decode_split.hip).
//
// One pass over the keys: with s = q . k, c = scale * log2 e and a running reference r per row,
//   p = exp2(c s - r),  l = sum p,  o = sum p v,  out = o / l,  lse = (r + log2 l) ln 2.
// Where a score exceeds r by more than kLazy, r is raised to the next whole number above it, and what has
// been summed is scaled by the power of two between (exact, in the bf16 weights too).  Past |r| = kFar
// whole numbers are as coarse as fp32 scores: such rows keep the maximum m itself, p = exp2(c (s - m)).
//
// A workgroup takes one KV head and a tile of 128 query rows, a row being (token, query head of the
// group), so that the G query heads of a KV head share every key read.  Its 4 wavefronts have 32 rows
// each and step through the keys 64 (4 pages) at a time.  Scores are computed transposed,
// S^T = K Q^T with v_mfma_f32_32x32x16_bf16, which leaves each lane 32 scores of ONE row (the other half
// of the row's 64 in lane ^ 32): maximum and sum are in-lane.  The weights, rounded to bf16, are the B
// operand of O^T = V^T P^T as they lie: the sum over keys may run in any order, so the keys of a step's
// 16 are taken in the order in which the scores' layout has them, and V is read from LDS in that order,
// transposed by ds_read_b64_tr_b16.  Rounding the weights to bf16 (2^-9 relative, to nearest, so errors
// average out over the keys) is what the matrix cores take; l sums the unrounded weights in fp32.
//
// A compute unit holds two workgroups (64 KB of LDS each for two steps' keys, 206 registers): one wavefront
// issues a vector instruction every 8 cycles at most, so two a SIMD are what it takes to weigh scores under the
// matrix instructions.  Measured: 4,096 tokens after 12,288 at 64/8 heads 1.73 to 1.81 ms, 1.07 to 1.11 PFLOP/s,
// the matrix cores busy 59% of the cycles and the vector ALUs 55%, at the 1.73 GHz that the power limit leaves
// (a library product of 16,384^3 reaches 1.64 PFLOP/s); up to 8 tokens of 4 requests over up to 36,480 positions
// at 32/8 heads 69 us, 5.3 TB/s of keys and values.  64 rows a wavefront, one workgroup of 512 registers (half
// the LDS reads a row), took 1.68 ms where this took 1.78, but longer on everything smaller; 8 wavefronts a
// workgroup with 4 buffers 1.84 against 1.86 ms and no less elsewhere; two groups of keys in a workgroup 10% less
// for some prompts of a few hundred tokens and more for most.
#pragma once

#include <float.h>
#include <math.h>

#include <type_traits>

#include "merge_body.h"
#include "qf_internal.h"
#include "row_owner.h"

namespace qf {
namespace rows {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int D = kHeadDim;
constexpr int P = kPage;
constexpr int W = 4;                     // wavefronts of a workgroup
constexpr int kRowsPerWave = kRowsTile / W;
constexpr int kPagesPerTile = kKeyTile / P;
constexpr int kTileBytes = kKeyTile * D * 2;
constexpr int kBufferBytes = 2 * kTileBytes;         // K and V of a step
constexpr int kUnit = kKeyTile / 2;                  // keys that the pipeline takes at a time
constexpr int kUnitBytes = kUnit * D * 2;
constexpr int kRing = 4;                             // fragments in registers
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLazy = 8.0f;            // log2 units: p <= 256 between rescales
constexpr float kFar = 1048576.0f;       // log2 units
// Steps of a key range, from what is known of all tiles of a KV head: `all` steps of `tiles` tiles, the longest
// of `longest`.  The least that fits the items and the entries fills the chip, but ranges cost too: a row's
// pair is 516 bytes written and read again, kRowsPairUs a range of all rows and heads, so a range is at least
// as long as minimises kRowsStepUs range + pair avg / range; and where no cut at all is faster, there is none:
//   uncut          kRowsAloneUs (with a workgroup to a compute unit, else kRowsStepUs) x longest
//   ranges         kRowsStepUs x range + kRowsJoinUs + pair (avg / range + 1/2)
// Measured (us, cut to fill the chip / uncut): 1,024 causal tokens at 16/8 heads 32.8 / 24.2, 2,048 54.7 /
// 44.1, 128 11.4 / 8.4, but 256 tokens after 4,096 32.2 / 81; 32 rows over 8,192 positions at 32/8 heads
// 14.6 with 4 steps a range, 16.6 with 3.
// Beside the sweep (no out) fewer items leave it room: half or all of the compute units without one, or half of
// what they hold, as long as the ranges stay short.  Whole calls with a quarter / half / all of the items, us:
// 32 requests over 8,192 positions at 32/8 heads (ranges of 9 / 5 / 5 steps) 26.6 / 31.8 / 32.7, 64 over 16,384
// (37 / 18 / 10) 61.0 / 56.2 / 64.7, 256 in 8 groups over up to 4,096 (64 / 22 / 10) 104.6 / 90.9 / 100.2, but
// 4 over 1,531 (2 / 1 / 1) 13.2 / 12.0 / 12.5 and 128 in 3 groups over up to 32,768 at 64/8 (-/ 126 / 53)
// 481 / 222 / 206-211.
__device__ __forceinline__ int range_of(const RowsParams& p, int64_t all, int64_t tiles, int longest) {
  if (tiles == 0) return 1;
  auto fits = [&](int64_t slots) {       // steps of a range with at most so many items
    return slots > tiles ? (all + slots - tiles - 1) / (slots - tiles) : (int64_t)INT32_MAX;
  };
  int64_t least = fits(p.slots);
  if (p.out == nullptr) {
    const int64_t quarter = fits(p.slots / 4), half = fits(p.slots / 2);
    if (quarter >= 4 && quarter <= 12) least = quarter;
    else if (half >= 4 && half <= 32) least = half;
  }
  least = max(least, (int64_t)((longest + p.entries - 1) / p.entries));
  const float avg = (float)all / (float)tiles, pair = kRowsPairUs * (float)p.rows * (float)p.hq;
  const int64_t range = max(least, (int64_t)ceilf(sqrtf(pair * avg / kRowsStepUs)));
  const float uncut = (tiles * p.hkv <= 256 ? kRowsAloneUs : kRowsStepUs) * (float)longest;
  const float cut = kRowsStepUs * (float)range + kRowsJoinUs + pair * (avg / (float)range + 0.5f);
  if (p.out != nullptr && uncut <= cut) return INT32_MAX;
  return (int)min(max(range, (int64_t)1), (int64_t)INT32_MAX);
}
static_assert(kPagesPerTile == W, "a wavefront stages one page of each step");

typedef const __attribute__((address_space(4))) int32_t* const_i32_ptr;

// 16-byte slot, within the 16 of its row, of chunk ch (dims 8 ch .. 8 ch + 7) of row i of a page in LDS.
// A row is 256 bytes, one round of the banks: the swizzle puts a chunk of 16 rows into 16 different
// slots (the score operand's reads) and 4 neighbouring chunks of 4 rows too (the transposed reads).
__device__ __forceinline__ int slot(int i, int ch) { return ch ^ (4 * (i & 3) + (i >> 2)); }

// The other half-wavefront's value of x (lane ^ 32).
__device__ __forceinline__ float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// One page (4 KB) from global memory straight to LDS, by one wavefront: load j takes rows 4 j .. 4 j + 3,
// lane l from page + 1024 j + (at ^ 16 j) to LDS byte to + 1024 j + 16 l.  Written as one block because the
// compiler, which cannot tell the LDS buffers apart, would wait for the loads before every transposed read
// of another buffer; whoever reads the page waits by hand (arrived()).  No output registers; M0 holds the
// LDS base, which the loads may follow after one wait state (the compiler reserves M0 and sets it before
// each use of its own).
__device__ __forceinline__ void load_page(const void* page, int at, uint32_t to) {
  asm volatile(
      "s_mov_b32 m0, %5\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %0\n\t"
      "global_load_lds_dwordx4 %2, %0 offset:1024\n\t"
      "global_load_lds_dwordx4 %3, %0 offset:2048\n\t"
      "global_load_lds_dwordx4 %4, %0 offset:3072"
      :
      : "s"(page), "v"(at), "v"(at ^ 16), "v"(at ^ 32), "v"(at ^ 48), "s"(to)
      : "memory");
}
// Every load of this wavefront has arrived; then every wavefront's.
__device__ __forceinline__ void arrived() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Sequence b: its rows (none where they are out of order or range) and the positions before them.
struct Sequence {
  int start, len, before;
  int poison;                            // a length out of range: no position is read
};
__device__ __forceinline__ Sequence sequence(const int32_t* __restrict__ cu,
                                             const int32_t* __restrict__ ctx_lens, int32_t rows,
                                             int32_t max_pages, bool causal, int b) {
  Sequence q{0, 0, 0, 0};
  const int s = cu[b], e = cu[b + 1], n = ctx_lens[b];
  if (s < 0 || e <= s || e > rows) return q;
  q.start = s;
  q.len = e - s;
  q.poison = n < 0 || (int64_t)n + (causal ? q.len : 0) > (int64_t)max_pages * P;
  q.before = q.poison ? 0 : n;
  return q;
}
// Positions that row `index` of it sees, and the steps of the tile whose first row (of len << gshift) is
// `first`: those of its last row.
__device__ __forceinline__ int sees_of(const Sequence& q, bool causal, int index) {
  return q.poison ? 0 : causal ? q.before + index + 1 : q.before;
}
__device__ __forceinline__ int keys_of(const Sequence& q, bool causal, int gshift, int first) {
  return sees_of(q, causal, min(first + kRowsTile - 1, (q.len << gshift) - 1) >> gshift);
}
__device__ __forceinline__ int steps_of(int keys) { return keys / kKeyTile + (keys % kKeyTile != 0); }
__device__ __forceinline__ int tiles_of(const Sequence& q, int gshift) {
  return (int)((((int64_t)q.len << gshift) + kRowsTile - 1) / kRowsTile);
}
// A tile's keys are cut into ranges of `range` steps.
__device__ __forceinline__ int ranges_of(int steps, int range) { return steps > 0 ? (steps - 1) / range + 1 : 1; }

// x combined over the lanes up to this one, six steps of DPP: rows of 16 first, then rows into later ones (a
// reduction by shuffles takes some 800 cycles through LDS, and a bisection below has ten).  `none`: of lanes that
// a step finds nothing for.
template <typename F>
__device__ __forceinline__ int upto(int x, int none, F f) {
  x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x111, 0xf, 0xf, false));      // row_shr:1, 2, 4, 8
  x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x112, 0xf, 0xf, false));
  x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x114, 0xf, 0xf, false));
  x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x118, 0xf, 0xf, false));
  x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x142, 0xa, 0xf, false));      // row_bcast:15
  return f(x, __builtin_amdgcn_update_dpp(none, x, 0x143, 0xc, 0xf, false));   // row_bcast:31
}
__device__ __forceinline__ int upto_sum(int x) {
  return upto(x, 0, [](int a, int b) { return a + b; });
}
// Over all lanes, in a scalar register.
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(upto_sum(x), 63); }
__device__ __forceinline__ int wave_max(int x) {
  return __builtin_amdgcn_readlane(upto(x, INT32_MIN, [](int a, int b) { return max(a, b); }), 63);
}
__device__ __forceinline__ int64_t wave_sum64(int64_t x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// What a workgroup does: rows first .. first + 127 of sequence seq, key range `part`.
struct Work {
  int seq, first, part, range;
  Sequence q;
};
// Tiles of a causal sequence with at least n steps: from the first on whose last row sees more than
// (n - 1) kKeyTile positions.
__device__ __forceinline__ int tiles_from(const Sequence& q, int gshift, int tiles, int n) {
  if (q.poison) return n <= 0 ? tiles : 0;
  const int64_t need = max((int64_t)0, (int64_t)(n - 1) * kKeyTile - q.before);   // rows before the first such
  if (need >= q.len) return 0;
  return tiles - (int)((need << gshift) / kRowsTile);
}
// The place among the tiles by length, the longest first, that slot takes.  A workgroup that starts late has to be
// short; and of the two that begin on a compute unit, the slot-th and the one `half` after it, one is as much
// longer than the middle as the other is shorter: the first half of the places go in reverse (one prompt, longest
// first in both halves -> so, us: 1,500 tokens at 32/8 heads 45.5 -> 40.1, 2,048 51.8 -> 49.4, 4,096 148 -> 142,
// 3,000 at 16/8 72 -> 66.5; from some thousand tiles on no difference).
__device__ __forceinline__ int length_rank(const RowsParams& p, int slot) {
  const int half = min(kRowsResident / 2 / p.hkv, p.slots);
  return slot < half ? half - 1 - slot : slot;
}

// Work item `slot` of a KV head.  The range (range_of) leaves at most p.slots items and p.entries ranges a
// tile: with t tiles of n steps each sequence has t ceil(n / range) of them.  Items of a range of keys lie
// side by side (their tiles read the same keys).  Causal tiles without ranges differ in length: they are taken
// by length (length_rank), found by bisection for the tile's number of steps, then among the tiles of just that
// many.
// At most 64 sequences: every wavefront finds it for itself, a lane to a sequence.
__device__ __forceinline__ Work find_among_few(const RowsParams& p, int gshift, int slot) {
  const int lane = threadIdx.x & 63;
  Sequence q{0, 0, 0, 0};
  if (lane < p.seqs) q = sequence(p.cu, p.ctx_lens, p.rows, p.max_pages, p.causal, lane);
  const int t = tiles_of(q, gshift);
  const int n = t > 0 ? steps_of(sees_of(q, p.causal, q.len - 1)) : 0;
  int range = INT32_MAX, above = 0;      // above: tiles of the sequence that are longer
  if (p.entries > 1) {
    const int64_t all = wave_sum64((int64_t)t * n);
    const int tiles = wave_sum(t), longest = wave_max(n);
    range = __builtin_amdgcn_readfirstlane(range_of(p, all, tiles, longest));
  }
  const bool by_length = p.causal && range == INT32_MAX;
  int before = 0, items;                 // at most 64 x 2^24 tiles; ranges only of few
  if (by_length) {
    slot = length_rank(p, slot);
    int low = 0, high = wave_max(n) + 1; // tiles of at least low, high steps: > slot (or none), <= slot
    while (high - low > 1) {
      const int mid = (low + high) / 2;
      if (wave_sum(tiles_from(q, gshift, t, mid)) > slot) low = mid; else high = mid;
    }
    above = tiles_from(q, gshift, t, low + 1);
    before = wave_sum(above);
    items = tiles_from(q, gshift, t, low) - above;
  } else {
    items = t * ranges_of(n, range);
  }
  const int end = before + upto_sum(items);
  const uint64_t past = __ballot(end > slot);
  if (past == 0) return Work{-1, 0, 0, range, Sequence{0, 0, 0, 0}};
  const int l = __builtin_ctzll(past);
  auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
  const int i = __builtin_amdgcn_readfirstlane(slot - of(end - items)), tl = of(t);
  const Sequence found{of(q.start), of(q.len), of(q.before), of(q.poison)};
  if (by_length) return Work{l, (tl - of(above) - 1 - i) * kRowsTile, 0, range, found};
  return Work{l, i % tl * kRowsTile, i / tl, range, found};
}

// More sequences: the workgroup together, thread t looking at sequences t, t + 256, ...; their items lie in
// order of (t, sequence).  Tiles of different lengths go by their number of bits of steps, the most first,
// counted in one pass.
struct Many {
  int64_t all[W], tiles[W];              // sums of each wavefront
  int longest[W];
  int tiles_of_bits[33];
  Work work;
};
__device__ __forceinline__ Work find_among_many(const RowsParams& p, int gshift, int slot, Many& lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int range = INT32_MAX, bits = 0;
  int64_t before = 0;
  auto each = [&](auto use) {            // this thread's sequences: their tiles, and steps of the longest
    for (int b = threadIdx.x; b < p.seqs; b += 64 * W) {
      const Sequence q = sequence(p.cu, p.ctx_lens, p.rows, p.max_pages, p.causal, b);
      const int t = tiles_of(q, gshift);
      use(b, q, t, t > 0 ? steps_of(sees_of(q, p.causal, q.len - 1)) : 0);
    }
  };
  // Tiles whose number of steps has at least k bits.
  auto with_bits = [&](const Sequence& q, int t, int k) {
    return k > 31 ? 0 : tiles_from(q, gshift, t, k == 0 ? 0 : 1 << (k - 1));
  };
  if (threadIdx.x == 0) lds.work = Work{-1, 0, 0, 0, Sequence{0, 0, 0, 0}};
  if (p.entries > 1) {
    int64_t all = 0, tiles = 0;
    int longest = 0;
    each([&](int, const Sequence&, int t, int n) {
      all += (int64_t)t * n;
      tiles += t;
      longest = max(longest, n);
    });
    all = wave_sum64(all);
    tiles = wave_sum64(tiles);
    longest = wave_max(longest);
    if (lane == 0) {
      lds.all[wave] = all;
      lds.tiles[wave] = tiles;
      lds.longest[wave] = longest;
    }
    __syncthreads();
    all = tiles = longest = 0;
    for (int w = 0; w < W; ++w) {
      all += lds.all[w];
      tiles += lds.tiles[w];
      longest = max(longest, lds.longest[w]);
    }
    range = __builtin_amdgcn_readfirstlane(range_of(p, all, tiles, longest));
  }
  const bool by_length = p.causal && range == INT32_MAX;
  if (by_length) {
    slot = length_rank(p, slot);
    if (threadIdx.x < 33) lds.tiles_of_bits[threadIdx.x] = 0;
    __syncthreads();
    each([&](int, const Sequence& q, int t, int n) {
      int longer = 0;
      for (int k = n > 0 ? 32 - __builtin_clz(n) : 0; longer < t && k >= 0; --k) {
        const int so_far = with_bits(q, t, k);
        if (so_far > longer) atomicAdd(&lds.tiles_of_bits[k], so_far - longer);
        longer = so_far;
      }
    });
    __syncthreads();
    const int items = lane < 33 ? lds.tiles_of_bits[32 - lane] : 0, end = upto_sum(items);
    const uint64_t past = __ballot(end > slot);
    if (past == 0) return Work{-1, 0, 0, range, Sequence{0, 0, 0, 0}};
    const int l = __builtin_ctzll(past);
    bits = __builtin_amdgcn_readfirstlane(32 - l);
    before = __builtin_amdgcn_readlane(end - items, l);
  }
  auto items_of = [&](const Sequence& q, int t, int n) {
    return by_length ? (int64_t)(with_bits(q, t, bits) - with_bits(q, t, bits + 1))
                     : (int64_t)t * ranges_of(n, range);
  };
  int64_t mine = 0;
  each([&](int, const Sequence& q, int t, int n) { mine += items_of(q, t, n); });
  // No call has 2^24 items; more, of ranges of rows that overlap, must not wrap to two owners of a slot.
  mine = min(mine, (int64_t)1 << 24);
  int64_t upto = upto_sum((int)mine);
  __syncthreads();                       // the sums above are read
  if (lane == 63) lds.all[wave] = upto;
  __syncthreads();
  upto += before;
  for (int w = 0; w < wave; ++w) upto += lds.all[w];
  int64_t at = slot - (upto - mine);     // among this thread's, in one thread of the workgroup
  if (at >= 0 && at < mine)
    each([&](int b, const Sequence& q, int t, int n) {
      const int64_t items = items_of(q, t, n);
      if (at >= 0 && at < items) {
        const int i = (int)at;
        lds.work = by_length ? Work{b, (t - with_bits(q, t, bits + 1) - 1 - i) * kRowsTile, 0, range, q}
                             : Work{b, i % t * kRowsTile, i / t, range, q};
      }
      at -= items;
    });
  __syncthreads();
  Work found = lds.work;
  found.range = range;
  __syncthreads();                       // read, before the keys take its place
  return found;
}

__device__ __forceinline__ Work find_work(const RowsParams& p, int gshift, int slot, Many& lds) {
  if (p.seqs > 64) return find_among_many(p, gshift, slot, lds);
  if (p.seqs > 1) return find_among_few(p, gshift, slot);
  // One: by scalar instructions alone; causal tiles grow longer with their number.
  const Sequence q = sequence((const int32_t*)(const_i32_ptr)p.cu, (const int32_t*)(const_i32_ptr)p.ctx_lens,
                              p.rows, p.max_pages, p.causal, 0);
  const int t = tiles_of(q, gshift);
  const int n = t > 0 ? steps_of(sees_of(q, p.causal, q.len - 1)) : 0;
  int range = INT32_MAX;
  if (p.entries > 1) range = __builtin_amdgcn_readfirstlane(range_of(p, (int64_t)t * n, t, n));
  const int parts = ranges_of(n, range);
  if (p.causal && range == INT32_MAX) {
    const int rank = length_rank(p, slot);
    return Work{rank < t ? 0 : -1, (t - 1 - rank) * kRowsTile, 0, range, q};
  }
  if (slot >= t * parts) return Work{-1, 0, 0, range, q};
  return Work{0, slot % t * kRowsTile, slot / t, range, q};
}

// A bf16 pair with zeros for infinities and NaN.
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}

// A workgroup's LDS: two steps' K and V (before them, what finds the work item), and whether V had infinities
// or NaN among masked steps.
struct Lds {
  union {
    alignas(1024) unsigned char kv[2 * kBufferBytes];
    Many many;
  };
  int found;
};

// Work item `item` of p (item % hkv: its KV head), by a whole workgroup.
__device__ __forceinline__ void item(const RowsParams& p, const unsigned item, Lds& lds_mem) {
  auto& s_kv = lds_mem.kv;
  int& s_found = lds_mem.found;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5;
  const int gshift = 31 - __builtin_clz(p.hq / p.hkv);

  const int g = item % (unsigned)p.hkv;
  Work work = find_work(p, gshift, item / (unsigned)p.hkv, lds_mem.many);
  for (int* x : {&work.seq, &work.first, &work.part, &work.range, &work.q.start, &work.q.len, &work.q.before,
                 &work.q.poison})
    *x = __builtin_amdgcn_readfirstlane(*x);       // equal in every lane: into scalar registers
  if (item == 0 && threadIdx.x == 0 && p.range != nullptr) *p.range = work.range;
  if (work.seq < 0) return;
  const int b = work.seq;
  const Sequence& seq = work.q;

  // This lane's row: token and query head; rows past the sequence's repeat its last one.
  const int n_rows = seq.len << gshift;
  const int row = work.first + wave * kRowsPerWave + (lane & 31);
  const bool live = row < n_rows;
  const int index = (live ? row : n_rows - 1) >> gshift;
  const int h = (g << gshift) + ((live ? row : n_rows - 1) & ((1 << gshift) - 1));
  const int64_t out_row = (int64_t)seq.start + index;

  // Positions that the row, every row of the wavefront, and some row of the tile sees.
  const bool poison = seq.poison;
  const int sees = sees_of(seq, p.causal, index);
  const int all_see =
      sees_of(seq, p.causal, min(work.first + wave * kRowsPerWave, n_rows - 1) >> gshift);
  const int keys = keys_of(seq, p.causal, gshift, work.first);
  const int steps = steps_of(keys);
  const int parts = ranges_of(steps, work.range);
  if (work.part >= parts) return;
  const int k0 = work.part * work.range;             // no overflow: < steps, or part 0
  const int k1 = (int)min((int64_t)k0 + work.range, (int64_t)steps);

  // The queries: B operand of S^T, lane (half, row) holds dims 16 kk + 8 half .. + 7.  A negative scale
  // is their sign; a zero one becomes 1e-37, so that scores of -inf stay -inf.
  bf16x8 q[8];
  {
    const uint4* src = reinterpret_cast<const uint4*>(p.q + (out_row * p.hq + h) * D);
    const uint32_t flip = p.scale_log2 < 0.0f ? 0x80008000u : 0u;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      uint4 w = src[2 * kk + half];
      w.x ^= flip; w.y ^= flip; w.z ^= flip; w.w ^= flip;
      q[kk] = __builtin_bit_cast(bf16x8, w);
    }
  }
  const float scale = fmaxf(fabsf(p.scale_log2), 1e-37f);

  f32x16 o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  // The reference starts at the lowest finite value: no difference is inf - inf.
  float m = -FLT_MAX, less = -FLT_MAX, l = 0.0f;   // less: the reference, 0 where m is it
  bool is_far = false, far = false;      // m is, for this row, for some row of the wavefront

  const int pages = (keys + P - 1) / P;
  const const_i32_ptr bt =
      p.block_table ? (const_i32_ptr)(p.block_table + (int64_t)b * p.max_pages) : nullptr;
  const int64_t head_off = (int64_t)g * P * D;
  const int64_t page_stride = (int64_t)p.hkv * P * D;

  // Lane addresses.  Scores: key 32 t + (lane & 31), chunk 2 kk + half.  V: lane group of 16 reads 4 keys
  // by 16 dims, key 8 r + 4 half + (lane & 15) / 4 of the step's 16, dims 32 d + 16 ((lane >> 4) & 1) + ...
  // Both are a lane's base with the chunk's higher bits exclusive-or'ed in (slot()).
  // They are kept, and toggled between the two buffers once a step.
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)s_kv;
  uint32_t ka[8], va[8];
  {
    const int kbase = (lane & 31) * (D * 2) + slot(lane & 15, half) * 16;
    const int vrow = 4 * half + ((lane & 15) >> 2);
    const int vbase = vrow * (D * 2) + slot(vrow, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) * 16 +
                      8 * (lane & 1);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) ka[kk] = lds0 + (kbase ^ (32 * kk));
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 2; ++r)
        va[2 * d + r] = lds0 + kTileBytes + 8 * r * (D * 2) + (vbase ^ (64 * d + 32 * r));
  }

  // A step's 4 pages go straight to LDS, one per wavefront.  The lanes' places there are consecutive, so
  // the swizzle is in the addresses that they read from.  A page past the last repeats it (its keys are
  // masked); one outside the pool is read as page 0 and its scores become NaN.
  const int at = (lane >> 4) * (D * 2) + ((lane & 15) ^ (4 * (lane >> 4))) * 16;
  struct Pages {
    int of[kPagesPerTile];
  };
  auto entries = [&](int kt) {           // of step kt, or of the last one
    Pages e;
#pragma unroll
    for (int j = 0; j < kPagesPerTile; ++j) e.of[j] = min(kt * kPagesPerTile + j, pages - 1);
    if (bt) {
#pragma unroll
      for (int j = 0; j < kPagesPerTile; ++j) e.of[j] = bt[e.of[j]];
    } else {
#pragma unroll
      for (int j = 0; j < kPagesPerTile; ++j) e.of[j] += b * p.max_pages;
    }
    return e;
  };
  const uint32_t lds = lds0 + wave * (P * D * 2);
  // This wavefront's page of a step; bit j of bad: page j is outside the pool.
  auto my_page = [&](const Pages& e, int& bad) {
    int mine = 0;
    bad = 0;
#pragma unroll
    for (int j = 0; j < kPagesPerTile; ++j) {
      const bool in = (unsigned)e.of[j] < (unsigned)p.num_pages;
      bad |= in ? 0 : 1 << j;
      if (j == wave) mine = in ? e.of[j] : 0;
    }
    return mine;
  };
  auto load_k = [&](int page, int to) { load_page(p.k + page * page_stride + head_off, at, lds + to); };
  auto load_v = [&](int page, int to) {
    load_page(p.v + page * page_stride + head_off, at, lds + to + kTileBytes);
  };

  // From step `edge` on, some row of the tile does not see every key.  A masked key's weight is 0, but 0
  // times an infinity or NaN is not: so every wavefront makes zeros of those in its page of V.  Where there
  // were any at a position of the request's (rare; what lies behind its last in the page is nobody's), they are
  // added at the end to the rows that do see them.
  const int edge = max(k0, sees_of(seq, p.causal, work.first >> gshift) / kKeyTile);
  auto clean = [&](int kt, int buffer) {
    unsigned char* const mine = s_kv + buffer + kTileBytes + wave * (P * D * 2);
    u32x4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = reinterpret_cast<const u32x4*>(mine)[64 * j + lane];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u32x4 y = {finite_pair(x[j].x), finite_pair(x[j].y), finite_pair(x[j].z), finite_pair(x[j].w)};
      if (((x[j].x ^ y.x) | (x[j].y ^ y.y) | (x[j].z ^ y.z) | (x[j].w ^ y.w)) != 0) {
        reinterpret_cast<u32x4*>(mine)[64 * j + lane] = y;
        if (kt * kKeyTile + wave * P + 4 * j + (lane >> 4) < keys) s_found = 1;
      }
    }
    __syncthreads();
  };

  // A fragment of K or V for one matrix instruction: of K (i < 8) the unit's 32 keys by dims 16 i .. + 15, of V
  // 16 keys by 32 dims.
  auto fragment = [&](int unit, int i) __attribute__((always_inline)) -> bf16x8 {
    if (i < 8)
      return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)(ka[i] + unit * kUnitBytes);
    const int d = i & 3, u = (i - 8) >> 2;
    s16x4 a[2];
#pragma unroll
    for (int r = 0; r < 2; ++r)
      a[r] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)(
          va[2 * d + r] + unit * kUnitBytes + 16 * u * (D * 2)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a[0], a[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // The highest of a unit's scores that the row sees.
  auto highest = [&](const f32x16& n) __attribute__((always_inline)) {
    float top = n[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, n[i]);
    return top;
  };
  // Scores n, from position key0 on, are next to be weighed, their highest being `top`: where some are masked
  // or in a bad page they are made so first, and where one is far above the reference, that is raised and
  // what was summed at the old one, weights w whose product is still to come among it, scaled.
  auto take = [&](f32x16& n, float top, u32x4 (&w)[2], int key0, int bad) __attribute__((always_inline)) {
    if (key0 + kUnit > all_see || bad != 0) {
      asm volatile("");                  // a branch, not 64 selections
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if ((bad >> (i / 8)) & 1) n[i] = NAN;
        if (key0 + 8 * (i / 4) + 4 * half + i % 4 >= sees) n[i] = -INFINITY;
      }
      top = highest(n);
    }
    top = fmaxf(top, other_half(top));
    if (!__any(fmaf(top, scale, -less) > kLazy) && !far) return;
    // The reference moves by whole numbers, so the factor is a power of two and exact in bf16 too.
    const float c_top = top * scale;
    const bool up = is_far ? (top - m) * scale > kLazy : c_top - less > kLazy;
    const bool now_far = up ? !(fabsf(c_top) <= kFar) : is_far;
    const float raised = up && !now_far ? ceilf(c_top) : less;
    const float f = !up ? 1.0f
                        : exp2f(is_far ? (m - top) * scale : less - (now_far ? c_top : raised));
    if (up) m = top;
    is_far = now_far;
    less = is_far ? 0.0f : raised;
    far = __any(is_far);
    l *= f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] *= f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x2 both = {(__bf16)(mrg::bf16_lo(w[u][i]) * f), (__bf16)(mrg::bf16_hi(w[u][i]) * f)};
        w[u][i] = __builtin_bit_cast(uint32_t, both);
      }
    if (is_far) {
#pragma unroll
      for (int i = 0; i < 16; ++i) n[i] -= m;
    }
  };
  // The weights of a unit in three stages of one vector instruction each: the exponent, the power, and its
  // place in the sum and (with the one before it) in a bf16 pair.  stage(i) is the third of weight i, the
  // second of i + 1 and the first of i + 2: none waits for another.  Pinned: the compiler would move them to
  // where the pairs are used, with twice the registers and away from the matrix instructions.
  float exponent[2], power[2], even = 0.0f;
  auto first_stage = [&](const f32x16& s, int i) __attribute__((always_inline)) {
    if (i < 16) exponent[i % 2] = fmaf(s[i], scale, -less);
  };
  auto second_stage = [&](int i) __attribute__((always_inline)) {
    if (i < 16) power[i % 2] = __builtin_amdgcn_exp2f(exponent[i % 2]);
  };
  auto begin_weights = [&](const f32x16& s) __attribute__((always_inline)) {
    first_stage(s, 0);
    first_stage(s, 1);
    second_stage(0);
  };
  auto stage = [&](const f32x16& s, int i, u32x4 (&w)[2]) __attribute__((always_inline)) {
    float e = power[i % 2];
    second_stage(i + 1);
    first_stage(s, i + 2);
    l += e;
    if (i % 2 == 0) {
      asm volatile("" : "+v"(e), "+v"(l), "+v"(power[(i + 1) % 2]), "+v"(exponent[i % 2]));
      even = e;
    } else {
      const bf16x2 both = {(__bf16)even, (__bf16)e};
      uint32_t bits = __builtin_bit_cast(uint32_t, both);
      asm volatile("" : "+v"(bits), "+v"(l), "+v"(power[(i + 1) % 2]), "+v"(exponent[i % 2]));
      w[i / 8][i % 8 / 2] = bits;
    }
  };
  auto weigh_all = [&](const f32x16& s, u32x4 (&w)[2]) __attribute__((always_inline)) {
    begin_weights(s);
#pragma unroll
    for (int i = 0; i < 16; ++i) stage(s, i, w);
  };
  auto score_part = [&](const bf16x8& a, int i, f32x16& n) __attribute__((always_inline)) {
    n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[i], n, 0, 0, 0);
  };
  auto product_part = [&](const bf16x8& a, int i, const u32x4 (&w)[2]) __attribute__((always_inline)) {
    o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
        a, __builtin_bit_cast(bf16x8, w[(i - 8) >> 2]), o[i & 3], 0, 0, 0);
  };
  // Unit `unit` of a step: the scores of the next step's unit (K at ka), the weights of the scores s, and the
  // product of the older weights w (V at va), none of which waits for another: 16 matrix instructions with
  // the vector instructions of one weight each between them, and the LDS reads kRing - 1 ahead.
  auto pipeline = [&](int unit, bf16x8 (&ring)[kRing], const f32x16& s, const u32x4 (&w)[2],
                      u32x4 (&now)[2], f32x16& n) __attribute__((always_inline)) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) n[i] = 0.0f;
    begin_weights(s);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int ahead = 16 * unit + i + kRing - 1;
      if (ahead < 32) ring[(i + kRing - 1) % kRing] = fragment(ahead / 16, ahead % 16);
      if (i < 8)
        score_part(ring[i % kRing], i, n);
      else
        product_part(ring[i % kRing], i, w);
      stage(s, i, now);
      // the highest score; n is complete after i = 7
      if (i == 9) top = fmaxf(fmaxf(n[0], n[1]), n[2]);
      if (i > 9) top = fmaxf(fmaxf(top, n[2 * i - 17]), n[2 * i - 16]);
      if (i == 15) top = fmaxf(top, n[15]);
      if (i >= 9) asm volatile("" : "+v"(top));      // here, not behind the branches
      __builtin_amdgcn_sched_barrier(0);
    }
    return top;
  };

  if (k0 < k1) {
    // K runs a step ahead of V: the wait for step kt is for K of kt + 1 and V of kt, and behind it K of
    // kt + 2 and V of kt + 1 are requested.
    int bad0 = 0, bad1 = 0, bad2 = 0;                // of steps kt, kt + 1, kt + 2
    int kt = k0, to = 0;                             // to: the buffer of kt
    int page = my_page(entries(kt), bad0);           // this wavefront's, of the K requested last
    load_k(page, 0);
    load_v(page, 0);
    if (kt + 1 < k1) {
      page = my_page(entries(kt + 1), bad1);
      load_k(page, kBufferBytes);
    }
    Pages next = entries(kt + 2);
    if (threadIdx.x == 0) s_found = 0;
    arrived();
    f32x16 s, n;
    u32x4 w[2] = {}, now[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = n[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) score_part(fragment(0, i), i, s);
    take(s, highest(s), w, kt * kKeyTile, bad0);
#pragma unroll
    for (int i = 0; i < 8; ++i) score_part(fragment(1, i), i, n);
    weigh_all(s, w);
    take(n, highest(n), w, kt * kKeyTile + kUnit, bad0 >> 2);
    s = n;
#pragma unroll
    for (int i = 0; i < 8; ++i) ka[i] ^= kBufferBytes;
    for (; kt + 1 < k1; ++kt) {
      arrived();                                     // K of kt + 1 and V of kt; older units are read
      load_v(page, to ^ kBufferBytes);
      bad2 = 0;
      if (kt + 2 < k1) {
        page = my_page(next, bad2);
        load_k(page, to);
        next = entries(kt + 3);
      }
      if (kt >= edge) clean(kt, to);
      bf16x8 ring[kRing];
#pragma unroll
      for (int i = 0; i < kRing - 1; ++i) ring[i] = fragment(0, i);
      float top = pipeline(0, ring, s, w, now, n);
      take(n, top, now, (kt + 1) * kKeyTile, bad1);
      top = pipeline(1, ring, n, now, w, s);
      take(s, top, w, (kt + 1) * kKeyTile + kUnit, bad1 >> 2);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ka[i] ^= kBufferBytes;
        va[i] ^= kBufferBytes;
      }
      bad1 = bad2;
      to ^= kBufferBytes;
    }
    arrived();
    if (kt >= edge) clean(kt, to);
    weigh_all(s, now);
#pragma unroll
    for (int i = 8; i < 16; ++i) product_part(fragment(0, i), i, w);
#pragma unroll
    for (int i = 8; i < 16; ++i) product_part(fragment(1, i), i, now);

    if (s_found != 0) {                              // infinities and NaN among the keys from `edge` on
#pragma unroll 1
      for (int pos = edge * kKeyTile; pos < (int)min((int64_t)keys, (int64_t)k1 * kKeyTile); ++pos) {
        const int entry = bt ? bt[pos / P] : b * p.max_pages + pos / P;
        if ((unsigned)entry >= (unsigned)p.num_pages) continue;    // its scores are NaN
        const uint16_t* const x = p.v + entry * page_stride + head_off + (pos % P) * D + 4 * half;
        if (pos >= sees) continue;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t v = x[32 * d + 8 * (i / 4) + i % 4];
            if ((v & 0x7f80u) == 0x7f80u) o[d][i] += mrg::bf16_lo(v);
          }
      }
    }
  }

  l += other_half(l);
  const bool empty = l == 0.0f;          // no position, or every score -inf
  const float inv = poison ? NAN : empty ? 0.0f : 1.0f / l;
  const float lse = poison ? NAN : empty ? -INFINITY : ((is_far ? m * scale : less) + log2f(l)) * kLn2;
  const bool to_pairs = parts > 1 || p.out == nullptr;
  if (live && half == 0) {
    if (to_pairs)
      p.part_lse[(out_row * p.entries + work.part) * p.hq + h] = lse;
    else if (p.lse != nullptr)
      p.lse[out_row * p.hq + h] = lse;
  }
  // A lane has 4 neighbouring dims of a row at a time; through LDS (the buffer that the last step is not
  // in, 8 KB a wavefront, swizzled as a page is) 16 lanes store 256 bytes of one.
  unsigned char* const swap =
      s_kv + (((k1 - k0) & 1) != 0 ? kBufferBytes : 0) + wave * (kRowsPerWave * D * 2);
  const int c = lane & 15;
  auto store = [&](auto to) {            // row 4 j + lane / 16 of the wavefront, to(its place, its chunk c)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 4 * j + (lane >> 4), at_row = work.first + wave * kRowsPerWave + r;
      const u32x4 x = *reinterpret_cast<const u32x4*>(swap + r * (D * 2) + (c ^ (r & 15)) * 16);
      const int64_t token = seq.start + (at_row >> gshift);
      if (at_row < n_rows) *to(token, (g << gshift) + (at_row & ((1 << gshift) - 1))) = x;
    }
  };
  const int mine = lane & 31;
  if (to_pairs) {
#pragma unroll
    for (int q2 = 0; q2 < 2; ++q2) {     // 64 dims at a time
#pragma unroll
      for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const f32x16& x = o[2 * q2 + d];
          *reinterpret_cast<float4*>(swap + mine * (D * 2) + ((8 * d + 2 * a + half) ^ (mine & 15)) * 16) =
              make_float4(x[4 * a] * inv, x[4 * a + 1] * inv, x[4 * a + 2] * inv, x[4 * a + 3] * inv);
        }
      store([&](int64_t token, int head) {
        return reinterpret_cast<u32x4*>(p.part_o + ((token * p.entries + work.part) * p.hq + head) * D) +
               16 * q2 + c;
      });
    }
  } else {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = empty && !poison ? 0.0f : o[d][4 * a + j] * inv;
        const bf16x2 lo = {(__bf16)x[0], (__bf16)x[1]}, hi = {(__bf16)x[2], (__bf16)x[3]};
        *reinterpret_cast<uint2*>(swap + mine * (D * 2) + ((4 * d + a) ^ (mine & 15)) * 16 + 8 * half) =
            make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
      }
    store([&](int64_t token, int head) {
      return reinterpret_cast<u32x4*>(p.out + (token * p.hq + head) * D) + c;
    });
  }
}

}  // namespace rows
}  // namespace qf
