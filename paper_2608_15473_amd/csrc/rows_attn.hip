// Attention of packed query rows over a paged grouped-query KV cache, on the matrix cores, and the join
// of the pairs that its key ranges leave.
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
#include <float.h>
#include <math.h>

#include <type_traits>

#include "merge_body.h"
#include "qf_internal.h"
#include "row_owner.h"

namespace qf {
namespace {

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

// The sequence and first row of a workgroup's tile; every wavefront computes it for itself.
struct Tile {
  int seq, start, len, first;            // first: index of its first row among the len * G of seq
};
__device__ __forceinline__ Tile find_tile(const int32_t* __restrict__ cu, int32_t seqs, int32_t rows,
                                          int gshift, int tile) {
  const int lane = threadIdx.x & 63;
  int before = 0;                        // tiles of the sequences before this round's
  for (int b0 = 0; b0 < seqs; b0 += 64) {
    const int b = b0 + lane;
    int start = 0, len = 0;
    if (b < seqs) {
      const int s = cu[b], e = cu[b + 1];
      if (s >= 0 && e > s && e <= rows) {
        start = s;
        len = e - s;
      }
    }
    const int n = (int)((((int64_t)len << gshift) + kRowsTile - 1) / kRowsTile);
    int upto = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    const uint64_t past = __ballot(before + upto > tile);
    if (past != 0) {
      const int l = __builtin_ctzll(past);
      const int end = __builtin_amdgcn_readlane(upto, l);
      const int nl = __builtin_amdgcn_readlane(n, l);
      return Tile{b0 + l, __builtin_amdgcn_readlane(start, l), __builtin_amdgcn_readlane(len, l),
                  (tile - before - (end - nl)) * kRowsTile};
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return Tile{-1, 0, 0, 0};
}

// A bf16 pair with zeros for infinities and NaN.
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}

__global__ void __launch_bounds__(64 * W, 2) rows_attn_kernel(const RowsParams p) {
  __shared__ __attribute__((aligned(1024))) unsigned char s_kv[2 * kBufferBytes];
  __shared__ int s_found;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5;
  const int gshift = 31 - __builtin_clz(p.hq / p.hkv);

  const unsigned bid = blockIdx.x;
  const int g = bid % p.hkv;
  const unsigned rest = bid / p.hkv;
  const Tile tile = find_tile(p.cu, p.seqs, p.rows, gshift, p.tiles - 1 - (int)(rest % p.tiles));
  const int split = rest / p.tiles;
  if (tile.seq < 0) return;
  const int b = tile.seq;

  // This lane's row: token and query head; rows past the sequence's repeat its last one.
  const int n_rows = tile.len << gshift;
  const int row = tile.first + wave * kRowsPerWave + (lane & 31);
  const bool live = row < n_rows;
  const int index = (live ? row : n_rows - 1) >> gshift;
  const int h = (g << gshift) + ((live ? row : n_rows - 1) & ((1 << gshift) - 1));
  const int64_t out_row = (int64_t)tile.start + index;

  // Positions that the row sees, and the most that any row of the tile does.
  const int64_t cap = (int64_t)p.max_pages * P;
  const int n0 = p.ctx_lens[b];
  const bool poison = n0 < 0 || (int64_t)n0 + (p.causal ? tile.len : 0) > cap;
  const int last_index = min(tile.first + kRowsTile - 1, n_rows - 1) >> gshift;
  const int sees = poison ? 0 : p.causal ? n0 + index + 1 : n0;
  const int keys = poison ? 0 : p.causal ? n0 + last_index + 1 : n0;
  // Every row of the wavefront sees at least this many positions.
  const int all_see = poison ? 0
                      : p.causal
                          ? n0 + (min(tile.first + wave * kRowsPerWave, n_rows - 1) >> gshift) + 1
                          : n0;
  const int steps = (keys + kKeyTile - 1) / kKeyTile;
  const int per = (steps + p.splits - 1) / p.splits;
  const int k0 = (int)min((int64_t)split * per, (int64_t)steps);
  const int k1 = min(k0 + per, steps);

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
  // were any (rare), they are added at the end to the rows that do see them.
  const int edge = max(k0, (poison ? 0 : p.causal ? n0 + (tile.first >> gshift) + 1 : n0) / kKeyTile);
  auto clean = [&](int buffer) {
    unsigned char* const mine = s_kv + buffer + kTileBytes + wave * (P * D * 2);
#pragma unroll 1
    for (int j = 0; j < 4; ++j) {
      uint4* const at4 = reinterpret_cast<uint4*>(mine + 1024 * j) + lane;
      const uint4 x = *at4;
      const uint4 y = make_uint4(finite_pair(x.x), finite_pair(x.y), finite_pair(x.z), finite_pair(x.w));
      if (((x.x ^ y.x) | (x.y ^ y.y) | (x.z ^ y.z) | (x.w ^ y.w)) != 0) {
        *at4 = y;
        s_found = 1;
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
  // Weights i and i + 1 of scores s, computed here and not where they are used next (they are kept as 8
  // registers, not the 16 that they are rounded from, and between the matrix instructions).
  auto weigh = [&](const f32x16& s, int i, u32x4 (&w)[2]) __attribute__((always_inline)) {
    const float e0 = __builtin_amdgcn_exp2f(fmaf(s[i], scale, -less));
    const float e1 = __builtin_amdgcn_exp2f(fmaf(s[i + 1], scale, -less));
    const bf16x2 both = {(__bf16)e0, (__bf16)e1};
    uint32_t bits = __builtin_bit_cast(uint32_t, both);
    l += e0;
    l += e1;
    asm volatile("" : "+v"(bits), "+v"(l));
    w[i / 8][i % 8 / 2] = bits;
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
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int ahead = 16 * unit + i + kRing - 1;
      if (ahead < 32) ring[(i + kRing - 1) % kRing] = fragment(ahead / 16, ahead % 16);
      if (i < 8)
        score_part(ring[i % kRing], i, n);
      else
        product_part(ring[i % kRing], i, w);
      if (i % 2 == 0) weigh(s, i, now);
      if (i == 10) top = fmaxf(n[0], n[1]);
      if (i >= 10 && i < 15)
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (2 + 3 * (i - 10) + j < 16) top = fmaxf(top, n[2 + 3 * (i - 10) + j]);
      if (i == 14) asm volatile("" : "+v"(top));     // here, not behind the branches
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
#pragma unroll
    for (int i = 0; i < 16; i += 2) weigh(s, i, w);
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
      if (kt >= edge) clean(to);
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
    if (kt >= edge) clean(to);
#pragma unroll
    for (int i = 0; i < 16; i += 2) weigh(s, i, now);
#pragma unroll
    for (int i = 8; i < 16; ++i) product_part(fragment(0, i), i, w);
#pragma unroll
    for (int i = 8; i < 16; ++i) product_part(fragment(1, i), i, now);

    if (s_found != 0) {                              // infinities and NaN among the keys from `edge` on
#pragma unroll 1
      for (int pos = edge * kKeyTile; pos < min(keys, k1 * kKeyTile); ++pos) {
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
  if (!live) return;
  const bool empty = l == 0.0f;          // no position, or every score -inf
  const float inv = empty ? 0.0f : 1.0f / l;
  const float lse = poison ? NAN : empty ? -INFINITY : ((is_far ? m * scale : less) + log2f(l)) * kLn2;
  if (p.part_o != nullptr) {
    const int64_t at = (out_row * p.splits + split) * p.hq + h;
    if (half == 0) p.part_lse[at] = lse;
    if (lse == -INFINITY) return;        // never read
    float4* dst = reinterpret_cast<float4*>(p.part_o + at * D);
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        dst[8 * d + 2 * a + half] = make_float4(o[d][4 * a] * inv, o[d][4 * a + 1] * inv,
                                                o[d][4 * a + 2] * inv, o[d][4 * a + 3] * inv);
  } else {
    const int64_t at = out_row * p.hq + h;
    if (half == 0 && p.lse != nullptr) p.lse[at] = lse;
    uint2* dst = reinterpret_cast<uint2*>(p.out + at * D);
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = poison ? NAN : empty ? 0.0f : o[d][4 * a + j] * inv;
        dst[8 * d + 2 * a + half] = make_uint2(mrg::bf16_rne(x[0]) | (mrg::bf16_rne(x[1]) << 16),
                                               mrg::bf16_rne(x[2]) | (mrg::bf16_rne(x[3]) << 16));
      }
  }
}

// One workgroup of J wavefronts per (row, head); groups of 16 entries, the first source's and then the
// second's, go round the wavefronts.
constexpr int J = 4;
__global__ void __launch_bounds__(64 * J) join_kernel(const JoinParams p) {
  const int row = blockIdx.x / p.hq, h = blockIdx.x % p.hq;
  const bool first = row_owner(p.cu, p.seqs, p.rows, row).seq >= 0;
  if (!first && p.b_entries == 0) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ga = first ? (p.a_entries + mrg::K - 1) / mrg::K : 0;
  const int gb = (p.b_entries + mrg::K - 1) / mrg::K;
  mrg::WaveMerge st;
  for (int i = wave; i < ga + gb; i += J) {
    const bool a = i < ga;
    const int entries = a ? p.a_entries : p.b_entries;
    const int e0 = (a ? i : i - ga) * mrg::K;
    const int n = min(mrg::K, entries - e0);
    const int64_t at = ((int64_t)row * entries + e0) * p.hq + h;
    const float* lse = (a ? p.a_lse : p.b_lse) + at;
    const float2* o = reinterpret_cast<const float2*>((a ? p.a_o : p.b_o) + at * D) + lane;
    const float x = lane < n ? lse[(int64_t)lane * p.hq] : -INFINITY;
    const uint64_t filled = __ballot(x != -INFINITY);
    float2 v[mrg::K];
#pragma unroll
    for (int k = 0; k < mrg::K; ++k)
      v[k] = (filled >> k) & 1 ? o[(int64_t)k * p.hq * (D / 2)] : make_float2(0.0f, 0.0f);
    st.add(x, v);
  }
  __shared__ mrg::WaveMergeLds<J> lds;
  lds.put(wave, lane, st);
  __syncthreads();
  if (wave != 0) return;
  float lse;
  const float2 o = lds.finish(0, J, lane, lse);
  const int64_t at = (int64_t)row * p.hq + h;
  if (p.pair)
    reinterpret_cast<float2*>(p.out)[at * (D / 2) + lane] = o;
  else
    reinterpret_cast<uint32_t*>(p.out)[at * (D / 2) + lane] =
        mrg::bf16_rne(o.x) | (mrg::bf16_rne(o.y) << 16);
  if (p.lse != nullptr && lane == 0) p.lse[at] = lse;
}

}  // namespace

hipError_t launch_rows_attn(const RowsParams& p, hipStream_t stream) {
  const unsigned grid = (unsigned)p.tiles * (unsigned)p.splits * (unsigned)p.hkv;
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL(rows_attn_kernel, dim3(grid), dim3(64 * W), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_join(const JoinParams& p, hipStream_t stream) {
  const unsigned grid = (unsigned)p.rows * (unsigned)p.hq;
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL(join_kernel, dim3(grid), dim3(64 * J), 0, stream, p);
  return hipGetLastError();
}

}  // namespace qf
