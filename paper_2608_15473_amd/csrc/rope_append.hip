// New tokens on their way into attention: queries and keys normalised per head and rotated by their
// positions, keys and values written into the paged cache.
//
// For token t of request b at position p = ctx_lens[b] + its index in the request, and every head:
//   n(x) = x / sqrt(mean_i x_i^2 + eps) * gain                 (or x, without a gain)
//   (x0, x1) -> a (x0 cos - x1 sin, x1 cos + x0 sin)           angle p * freqs[i], i < rotary / 2
// over the pairs (i, i + rotary / 2) or (2i, 2i + 1); the other dims of a head pass.  All in fp32 from
// bf16 inputs, one rounding per output.  The angle is p * freqs[i] in fp64, reduced there to a fraction
// of a turn: at position 2^20 an fp32 product would be off by 0.03 rad.
#include "merge_body.h"
#include "qf_internal.h"
#include "row_owner.h"

namespace qf {
namespace {

constexpr int D = kHeadDim;
constexpr int P = kPage;
constexpr int kThreads = 256;

__device__ __forceinline__ void unpack8(const uint4& w, float* f) {
  f[0] = mrg::bf16_lo(w.x); f[1] = mrg::bf16_hi(w.x);
  f[2] = mrg::bf16_lo(w.y); f[3] = mrg::bf16_hi(w.y);
  f[4] = mrg::bf16_lo(w.z); f[5] = mrg::bf16_hi(w.z);
  f[6] = mrg::bf16_lo(w.w); f[7] = mrg::bf16_hi(w.w);
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  auto pair = [&](int j) { return mrg::bf16_rne(f[j]) | (mrg::bf16_rne(f[j + 1]) << 16); };
  return make_uint4(pair(0), pair(2), pair(4), pair(6));
}

// One workgroup per token; 16 lanes per head, lane c holding dims 8c .. 8c + 7.
__global__ void __launch_bounds__(kThreads) rope_append_kernel(const RopeAppendParams p) {
  __shared__ float s_cos[D / 2], s_sin[D / 2];
  const int t = blockIdx.x;
  const RowOwner own = row_owner(p.cu_tokens, p.batch, p.tokens, t);
  if (own.seq < 0) return;                     // a row of no request: left as it is
  const int b = own.seq;
  const int64_t pos = (int64_t)p.ctx_lens[b] + own.index;
  const int half = p.rotary / 2;
  if ((int)threadIdx.x < half) {
    const double turns = (double)pos * (p.freqs[threadIdx.x] * 0.15915494309189535);
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    s_cos[threadIdx.x] = c * p.amplitude;
    s_sin[threadIdx.x] = s * p.amplitude;
  }
  // Where the token's key and value go; -1: nowhere (past the table, or a page outside the pool).
  int64_t row0 = -1;
  if (p.k != nullptr) {
    if (p.ctx_lens[b] >= 0 && pos < (int64_t)p.max_pages * P) {
      const int64_t entry = (int64_t)b * p.max_pages + pos / P;
      const int page = p.block_table ? p.block_table[entry] : (int)entry;
      if ((unsigned)page < (unsigned)p.num_pages)
        row0 = ((int64_t)page * p.hkv * P + pos % P) * D;
    }
    if (row0 < 0 && p.status && threadIdx.x == 0) *p.status = 1;
  }
  __syncthreads();

  const int lane = threadIdx.x & 63;
  const int c = threadIdx.x & 15;
  const int nq = p.q ? p.hq : 0, nk = p.k ? p.hkv : 0;
  for (int r0 = 0; r0 < nq + 2 * nk; r0 += kThreads / 16) {
    const int r = r0 + (int)threadIdx.x / 16;
    const bool in = r < nq + 2 * nk;
    const bool is_q = r < nq, is_v = r >= nq + nk;
    const int h = is_q ? r : is_v ? r - nq - nk : r - nq;
    const uint16_t* src = is_q   ? p.q + (int64_t)t * p.q_stride
                          : is_v ? p.v + (int64_t)t * p.v_stride
                                 : p.k + (int64_t)t * p.k_stride;
    uint4 w = make_uint4(0, 0, 0, 0);
    if (in) w = reinterpret_cast<const uint4*>(src + (int64_t)h * D)[c];
    if (!is_v) {
      float x[8];
      unpack8(w, x);
      const uint16_t* gain = is_q ? p.q_gain : p.k_gain;
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
      ss = mrg::row_sum16(ss);
      if (gain != nullptr) {
        const float n = 1.0f / sqrtf(ss * (1.0f / D) + p.eps);
        float g[8];
        unpack8(reinterpret_cast<const uint4*>(gain)[c], g);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * n * g[e];
      }
      if (p.interleaved) {
        if (8 * c < p.rotary) {
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const float cs = s_cos[4 * c + e / 2], sn = s_sin[4 * c + e / 2];
            const float a = x[e], d = x[e + 1];
            x[e] = fmaf(a, cs, -d * sn);
            x[e + 1] = fmaf(d, cs, a * sn);
          }
        }
      } else {
        // rotary is a multiple of 16: a pair's members are in lanes rotary / 16 apart, at one place
        const int step = p.rotary / 16;
        const bool second = c >= step;
        const int from = lane + (c >= 2 * step ? 0 : second ? -step : step);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = __shfl(x[e], from);
          if (c < 2 * step) {
            const int i = 8 * (second ? c - step : c) + e;
            const float sn = s_sin[i];
            x[e] = fmaf(x[e], s_cos[i], second ? y * sn : -y * sn);
          }
        }
      }
      w = pack8(x);
    }
    if (!in) continue;
    if (is_q)
      reinterpret_cast<uint4*>(p.q_out + ((int64_t)t * p.hq + h) * D)[c] = w;
    else if (row0 >= 0)
      reinterpret_cast<uint4*>((is_v ? p.v_cache : p.k_cache) + row0 + (int64_t)h * P * D)[c] = w;
  }
}

}  // namespace

hipError_t launch_rope_append(const RopeAppendParams& p, hipStream_t stream) {
  if (p.tokens == 0) return hipSuccess;
  hipLaunchKernelGGL(rope_append_kernel, dim3(p.tokens), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace qf
