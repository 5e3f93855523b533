// Launches of the rows' attention (rows_body.h), and the join of the pairs that its key ranges leave.
#include "merge_body.h"
#include "rows_body.h"

namespace qf {
namespace {

constexpr int D = kHeadDim;

__global__ void __launch_bounds__(64 * rows::W, 2) rows_attn_kernel(const RowsParams p) {
  __shared__ rows::Lds lds;
  rows::item(p, blockIdx.x, lds);
}

// Ranges that the pairs of a row lie in; 0: of no sequence.
__device__ __forceinline__ int parts_of(const JoinParams& p, int row) {
  const int gshift = 31 - __builtin_clz(p.hq / p.hkv);
  const RowOwner own = row_owner(p.cu, p.seqs, p.rows, row);
  if (own.seq < 0) return 0;
  const rows::Sequence q = rows::sequence(p.cu, p.ctx_lens, p.rows, p.max_pages, p.causal, own.seq);
  const int first = (own.index << gshift) / kRowsTile * kRowsTile;
  return min(rows::ranges_of(rows::steps_of(rows::keys_of(q, p.causal, gshift, first)), *p.range),
             p.a_entries);
}

// Groups of 16 entries, the first source's (`parts` of them) and then the second's: i, i + step, ...
__device__ __forceinline__ void add_pairs(const JoinParams& p, int row, int h, int parts, int i, int step,
                                          mrg::WaveMerge& st) {
  const int lane = threadIdx.x & 63;
  const int ga = (parts + mrg::K - 1) / mrg::K;
  const int gb = (p.b_entries + mrg::K - 1) / mrg::K;
  for (; i < ga + gb; i += step) {
    const bool a = i < ga;
    const int entries = a ? p.a_entries : p.b_entries;
    const int e0 = (a ? i : i - ga) * mrg::K;
    const int n = min(mrg::K, (a ? parts : entries) - e0);
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
}
__device__ __forceinline__ void write_joined(const JoinParams& p, int row, int h, float2 o, float lse) {
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)row * p.hq + h;
  if (p.pair)
    reinterpret_cast<float2*>(p.out)[at * (D / 2) + lane] = o;
  else
    reinterpret_cast<uint32_t*>(p.out)[at * (D / 2) + lane] =
        mrg::bf16_rne(o.x) | (mrg::bf16_rne(o.y) << 16);
  if (p.lse != nullptr && lane == 0) p.lse[at] = lse;
}

constexpr int J = 4;                     // wavefronts of a workgroup
// Few rows: one workgroup per (row, head), the groups of entries going round its wavefronts.
__global__ void __launch_bounds__(64 * J) join_wide_kernel(const JoinParams p) {
  const int row = blockIdx.x / p.hq, h = blockIdx.x % p.hq;
  const int parts = parts_of(p, row);
  if (p.b_entries == 0 && parts <= 1) return;        // no row, or one that is written already
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  mrg::WaveMerge st;
  add_pairs(p, row, h, parts, wave, J, st);
  __shared__ mrg::WaveMergeLds<J> lds;
  lds.put(wave, lane, st);
  __syncthreads();
  if (wave != 0) return;
  float lse;
  const float2 o = lds.finish(0, J, lane, lse);
  write_joined(p, row, h, o, lse);
}

// Many rows: a wavefront per (row, head), `split` workgroups a row, so that more of them are on their way at
// a time (128 rows of 64 heads 21.5 -> 15.3 us), and a row that needs nothing costs few workgroups.
__global__ void __launch_bounds__(64 * J) join_kernel(const JoinParams p, const int32_t split) {
  const int row = blockIdx.x / split;
  const int parts = parts_of(p, row);
  if (p.b_entries == 0 && parts <= 1) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  __shared__ mrg::WaveMergeLds<J> lds;
  for (int h = blockIdx.x % split * J + wave; h < p.hq; h += split * J) {
    mrg::WaveMerge st;
    add_pairs(p, row, h, parts, 0, 1, st);
    lds.put(wave, lane, st);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");     // LDS operations of a wavefront stay in order
    float lse;
    const float2 o = lds.finish(wave, 1, lane, lse);
    write_joined(p, row, h, o, lse);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

}  // namespace

hipError_t launch_rows_attn(const RowsParams& p, hipStream_t stream) {
  const unsigned grid = (unsigned)p.slots * (unsigned)p.hkv;
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL(rows_attn_kernel, dim3(grid), dim3(64 * rows::W), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_join(const JoinParams& p, hipStream_t stream) {
  const unsigned grid = (unsigned)p.rows * (unsigned)p.hq;
  if (grid == 0) return hipSuccess;
  if (grid < 2048) {
    hipLaunchKernelGGL(join_wide_kernel, dim3(grid), dim3(64 * J), 0, stream, p);
  } else {
    // As many workgroups a row as make 2,048 of them (8 a compute unit), each of J heads at least.
    const unsigned most = ((unsigned)p.hq + J - 1) / J, want = (2048u + (unsigned)p.rows - 1) / (unsigned)p.rows;
    const unsigned split = want < most ? want : most;
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)p.rows * split), dim3(64 * J), 0, stream, p, (int32_t)split);
  }
  return hipGetLastError();
}

}  // namespace qf
