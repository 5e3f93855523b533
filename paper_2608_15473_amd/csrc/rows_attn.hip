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

// One workgroup of J wavefronts per (row, head); groups of 16 entries, the first source's and then the
// second's, go round the wavefronts.
template <int J>
__global__ void __launch_bounds__(64 * J) join_kernel(const JoinParams p) {
  const int row = blockIdx.x / p.hq, h = blockIdx.x % p.hq;
  const int gshift = 31 - __builtin_clz(p.hq / p.hkv);
  const RowOwner own = row_owner(p.cu, p.seqs, p.rows, row);
  int parts = 0;                         // ranges of the row's tile
  if (own.seq >= 0) {
    const rows::Sequence q = rows::sequence(p.cu, p.ctx_lens, p.rows, p.max_pages, p.causal, own.seq);
    const int first = (own.index << gshift) / kRowsTile * kRowsTile;
    parts = min(rows::ranges_of(rows::steps_of(rows::keys_of(q, p.causal, gshift, first)), *p.range), p.a_entries);
  }
  if (p.b_entries == 0 && parts <= 1) return;        // no row, or one that is written already
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ga = (parts + mrg::K - 1) / mrg::K;
  const int gb = (p.b_entries + mrg::K - 1) / mrg::K;
  mrg::WaveMerge st;
  for (int i = wave; i < ga + gb; i += J) {
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
  const unsigned grid = (unsigned)p.slots * (unsigned)p.hkv;
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL(rows_attn_kernel, dim3(grid), dim3(64 * rows::W), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_join(const JoinParams& p, hipStream_t stream) {
  const unsigned grid = (unsigned)p.rows * (unsigned)p.hq;
  if (grid == 0) return hipSuccess;
  // Many rows: one wavefront each, so that more of them are on their way at a time; few: the entries side
  // by side.
  if (grid >= 2048)
    hipLaunchKernelGGL((join_kernel<1>), dim3(grid), dim3(64), 0, stream, p);
  else
    hipLaunchKernelGGL((join_kernel<4>), dim3(grid), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace qf
