// Attention of packed query rows over a paged grouped-query KV cache, on the matrix cores, and the join
// of the pairs that its key ranges leave.
//
// One pass over the keys with a running maximum m of s = q . k and a sum l per row, c = scale * log2 e:
//   p = exp2(c s - c m),  l = sum p,  o = sum p v,  out = o / l,  lse = (c m + log2 l) ln 2;
// when c s exceeds c m by more than kLazy, m is raised and l, o scaled by exp2(c m_old - c m_new).  One
// fused multiply-add makes c s - (c m rounded); all p of a row share the rounding's factor, so it cancels,
// but past |c m| = kFar it could overflow, and p is exp2(c (s - m)) from then on.
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
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLazy = 8.0f;            // log2 units: p <= 256 between rescales
constexpr float kFar = 1048576.0f;       // log2 units: up to here c m is rounded by 2^-4 at most
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

// One page of K and one of V (4 KB each) from global memory straight to LDS, by one wavefront: load j takes
// rows 4 j .. 4 j + 3, lane l from page + 1024 j + at[j] to LDS byte to + 1024 j + 16 l.  Written as one
// block because the compiler, which cannot tell the two LDS buffers apart, would wait for the loads before
// every transposed read of the other buffer; whoever reads the page waits by hand (arrived()).  No output
// registers; M0 holds the LDS base, which the loads may follow after one wait state (the compiler reserves
// M0 and sets it before each use of its own).
__device__ __forceinline__ void load_page(const void* k, const void* v, const int (&at)[4], uint32_t to) {
  asm volatile(
      "s_mov_b32 m0, %6\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %0\n\t"
      "global_load_lds_dwordx4 %3, %0 offset:1024\n\t"
      "global_load_lds_dwordx4 %4, %0 offset:2048\n\t"
      "global_load_lds_dwordx4 %5, %0 offset:3072\n\t"
      "s_mov_b32 m0, %7\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %1\n\t"
      "global_load_lds_dwordx4 %3, %1 offset:1024\n\t"
      "global_load_lds_dwordx4 %4, %1 offset:2048\n\t"
      "global_load_lds_dwordx4 %5, %1 offset:3072"
      :
      : "s"(k), "s"(v), "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "s"(to), "s"(to + kTileBytes)
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

__device__ __forceinline__ bool bad_pair(uint32_t w) {   // a bf16 of the pair is infinite or NaN
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}

__global__ void __launch_bounds__(64 * W, 2) rows_attn_kernel(const RowsParams p) {
  __shared__ __attribute__((aligned(1024))) unsigned char s_kv[4 * kTileBytes];   // 2 x (K, V)
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
  // m starts at the lowest finite value, and so does cm = c m: no difference is inf - inf.
  float m = -FLT_MAX, cm = -FLT_MAX, l = 0.0f;
  bool far = false;                      // wavefront-uniform: some row is past kFar

  const int pages = (keys + P - 1) / P;
  const const_i32_ptr bt =
      p.block_table ? (const_i32_ptr)(p.block_table + (int64_t)b * p.max_pages) : nullptr;
  const int64_t head_off = (int64_t)g * P * D;
  const int64_t page_stride = (int64_t)p.hkv * P * D;

  // Lane addresses.  Scores: key 32 t + (lane & 31), chunk 2 kk + half.  V: lane group of 16 reads 4 keys
  // by 16 dims, key 8 r + 4 half + (lane & 15) / 4 of the step's 16, dims 32 d + 16 ((lane >> 4) & 1) + ...
  // Both are a lane's base with the chunk's higher bits exclusive-or'ed in (slot()).
  const int kbase = (lane & 31) * (D * 2) + slot(lane & 15, half) * 16;
  const int vrow = 4 * half + ((lane & 15) >> 2);
  const int vbase = kTileBytes + vrow * (D * 2) +
                    slot(vrow, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) * 16 + 8 * (lane & 1);

  // A step's 4 pages go straight to LDS, one per wavefront.  The lanes' places there are consecutive, so
  // the swizzle is in the addresses that they read from.  A page past the last repeats it (its keys are
  // masked); one outside the pool is read as page 0 and its scores become NaN.
  int at[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    at[j] = (lane >> 4) * (D * 2) + ((lane & 15) ^ (4 * (lane >> 4) + j)) * 16;
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
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)s_kv +
                       wave * (P * D * 2);
  // Returns which pages of the step are outside the pool (bit j: page j).
  auto stage = [&](const Pages& e, int buffer) {
    int bad = 0, mine = 0;
#pragma unroll
    for (int j = 0; j < kPagesPerTile; ++j) {
      const bool in = (unsigned)e.of[j] < (unsigned)p.num_pages;
      bad |= in ? 0 : 1 << j;
      if (j == wave) mine = in ? e.of[j] : 0;
    }
    const int64_t off = mine * page_stride + head_off;
    load_page(p.k + off, p.v + off, at, lds + buffer * 2 * kTileBytes);
    return bad;
  };

  // One step on the keys in `kv`.  MASKED: some row of the wavefront does not see all of them, or a page is
  // outside the pool.
  auto step = [&](auto masked, int kt, const unsigned char* kv, int bad) {
    constexpr bool MASKED = decltype(masked)::value;
    // S^T of 2 x 32 keys.
    f32x16 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(kv + t * 32 * D * 2 + (kbase ^ (32 * kk)));
        s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[kk], s[t], 0, 0, 0);
      }
    }
    if constexpr (MASKED) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if ((bad >> (2 * t + i / 8)) & 1) s[t][i] = NAN;
          if (kt * kKeyTile + 32 * t + 8 * (i / 4) + 4 * half + i % 4 >= sees) s[t][i] = -INFINITY;
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) top = fmaxf(top, s[i / 16][i % 16]);
    top = fmaxf(top, other_half(top));
    if (__any((top - m) * scale > kLazy)) {
      const float raised = fmaxf(m, top), c_raised = fmaxf(raised * scale, -FLT_MAX);
      far = far || __any(fabsf(c_raised) > kFar && raised > -FLT_MAX);
      const float f = exp2f(far ? (m - raised) * scale : cm - c_raised);
      m = raised;
      cm = c_raised;
      l *= f;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= f;
    }
    if (far) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] -= m;
    }
    const float less = far ? 0.0f : cm;
    bf16x8 w[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[t][i], scale, -less));
        l += e;
        w[2 * t + i / 8][i % 8] = (__bf16)e;
      }

    // O^T += V^T P^T.
    bool unclean = false;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        uint2 a[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const unsigned char* from = kv + (16 * u + 8 * r) * (D * 2) + (vbase ^ (64 * d + 32 * r));
          a[r] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4*)from));
        }
        if constexpr (MASKED) {          // a masked key's weight is 0, but 0 times infinity is not
          unclean = unclean || bad_pair(a[0].x) || bad_pair(a[0].y) || bad_pair(a[1].x) || bad_pair(a[1].y);
          a[0] = make_uint2(finite_pair(a[0].x), finite_pair(a[0].y));
          a[1] = make_uint2(finite_pair(a[1].x), finite_pair(a[1].y));
        }
        const uint4 both = make_uint4(a[0].x, a[0].y, a[1].x, a[1].y);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, both), w[u], o[d],
                                                       0, 0, 0);
      }
    }
    if constexpr (MASKED) {
      if (!__any(unclean)) return;
      // Rare: the infinities and NaN of the keys that a row does see.
#pragma unroll 1
      for (int key = 0; key < kKeyTile; ++key) {
        const int i = key & 15;
        const bool seen = kt * kKeyTile + key < sees;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int dim = 32 * d + 8 * (e / 4) + 4 * half + e % 4;
            const uint32_t x = *reinterpret_cast<const uint16_t*>(
                kv + kTileBytes + key * (D * 2) + slot(i, dim / 8) * 16 + (dim % 8) * 2);
            if (seen && (x & 0x7f80u) == 0x7f80u) o[d][e] += mrg::bf16_lo(x);
          }
      }
    }
  };

  if (k0 < k1) {
    int bad = stage(entries(k0), 0), bad_now = 0, kt = k0;
    Pages next = entries(k0 + 1);
    // Waits for step kt and requests the next one; returns the keys.
    auto advance = [&]() -> const unsigned char* {
      const int buffer = (kt - k0) & 1;
      bad_now = bad;
      arrived();                         // the step's keys are here, and the last step's reads are done
      if (kt + 1 < k1) {
        bad = stage(next, 1 - buffer);
        next = entries(kt + 2);
      }
      return s_kv + buffer * 2 * kTileBytes;
    };
    while (kt < k1) {
      for (; kt < k1 && (kt + 1) * kKeyTile <= all_see && bad == 0; ++kt) {
        const unsigned char* const kv = advance();
        step(std::false_type{}, kt, kv, 0);
      }
      if (kt == k1) break;
      const unsigned char* const kv = advance();
      step(std::true_type{}, kt, kv, bad_now);
      ++kt;
    }
  }

  l += other_half(l);
  if (!live) return;
  const bool empty = l == 0.0f;          // no position, or every score -inf
  const float inv = empty ? 0.0f : 1.0f / l;
  const float lse = poison ? NAN : empty ? -INFINITY : (cm + log2f(l)) * kLn2;
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
        for (int j = 0; j < 4; ++j) x[j] = poison ? NAN : o[d][4 * a + j] * inv;
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
