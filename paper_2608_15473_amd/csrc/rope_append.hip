// New tokens on their way into attention: queries and keys normalised per head and rotated by their
// positions, keys and values written into the paged cache.
//
// For token t of request b at position p = ctx_lens[b] + its index in the request, and every head:
//   n(x) = x / sqrt(mean_i x_i^2 + eps) * gain                 (or x, without a gain)
//   (x0, x1) -> a (x0 cos - x1 sin, x1 cos + x0 sin)           angle p * freqs[i], i < rotary / 2
// over the pairs (i, i + rotary / 2) or (2i, 2i + 1); the other dims of a head pass.  All in fp32 from
// bf16 inputs, one rounding per output.  The angle is p * freqs[i] in fp64, reduced there to a fraction
// of a turn: at position 2^20 an fp32 product would be off by 0.03 rad.
//
// Bound by bytes, each read and written once: 17,437 tokens of 80 heads 140 us, 5.1 TB/s read and
// written together (a large device copy reaches 4.9); a step's single tokens by the launch, 3.2 to 4.2 us.
#include "merge_body.h"
#include "qf_internal.h"
#include "row_owner.h"

namespace qf {
namespace {

constexpr int D = kHeadDim;
constexpr int P = kPage;

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

// One workgroup of T threads per token; 16 lanes per head, lane c holding dims 8c .. 8c + 7, T / 16 heads
// at a time.  What a single token waits for is a chain of loads (the request's length, the page's number)
// and the angles: the first heads and the gains are requested before it.
template <int T>
__global__ void __launch_bounds__(T) rope_append_kernel(const RopeAppendParams p) {
  __shared__ float s_cos[D / 2], s_sin[D / 2];
  const int t = blockIdx.x;
  const int lane = threadIdx.x & 63;
  const int c = threadIdx.x & 15;
  const int nq = p.q ? p.hq : 0, nk = p.k ? p.hkv : 0, heads = nq + 2 * nk;
  auto load = [&](int r) {               // this lane's dims of head r: queries, then keys, then values
    if (r >= heads) return make_uint4(0, 0, 0, 0);
    const uint16_t* src = r < nq        ? p.q + (int64_t)t * p.q_stride + (int64_t)r * D
                          : r < nq + nk ? p.k + (int64_t)t * p.k_stride + (int64_t)(r - nq) * D
                                        : p.v + (int64_t)t * p.v_stride + (int64_t)(r - nq - nk) * D;
    return reinterpret_cast<const uint4*>(src)[c];
  };
  const int r0 = (int)threadIdx.x / 16;
  uint4 next = load(r0);
  uint4 q_gain = make_uint4(0, 0, 0, 0), k_gain = q_gain;
  if (p.q_gain != nullptr) q_gain = reinterpret_cast<const uint4*>(p.q_gain)[c];
  if (p.k_gain != nullptr) k_gain = reinterpret_cast<const uint4*>(p.k_gain)[c];
  const int half = p.rotary / 2;
  double freq = 0.0;
  if ((int)threadIdx.x < half) freq = p.freqs[threadIdx.x] * 0.15915494309189535;   // turns

  const RowOwner own = row_owner(p.cu_tokens, p.batch, p.tokens, t);
  if (own.seq < 0) return;               // a row of no request: left as it is
  const int b = own.seq;
  const int n = p.ctx_lens[b];
  const int64_t pos = (int64_t)n + own.index;
  // Where the token's key and value go; -1: nowhere (past the table, or a page outside the pool).
  int64_t row0 = -1;
  if (nk > 0) {
    if (n >= 0 && pos < (int64_t)p.max_pages * P) {
      const int64_t entry = (int64_t)b * p.max_pages + pos / P;
      const int page = p.block_table ? p.block_table[entry] : (int)entry;
      if ((unsigned)page < (unsigned)p.num_pages)
        row0 = ((int64_t)page * p.hkv * P + pos % P) * D;
    }
    if (row0 < 0 && p.status && threadIdx.x == 0) *p.status = 1;
  }
  if ((int)threadIdx.x < half) {
    const double turns = (double)pos * freq;
    float s, cs;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &cs);
    s_cos[threadIdx.x] = cs * p.amplitude;
    s_sin[threadIdx.x] = s * p.amplitude;
  }
  __syncthreads();

  for (int r = r0; r < (heads + 3) / 4 * 4; r += T / 16) {   // by whole wavefronts
    const bool is_q = r < nq, is_v = r >= nq + nk;
    uint4 w = next;
    next = load(r + T / 16);
    if (!is_v) {
      float x[8];
      unpack8(w, x);
      if (is_q ? p.q_gain != nullptr : p.k_gain != nullptr) {
        float ss = 0.0f, gain[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
        ss = mrg::row_sum16(ss);
        const float inv = 1.0f / sqrtf(ss * (1.0f / D) + p.eps);
        unpack8(is_q ? q_gain : k_gain, gain);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * gain[e];
      }
      if (p.interleaved) {
        if (8 * c < p.rotary) {
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const float cs = s_cos[4 * c + e / 2], sn = s_sin[4 * c + e / 2];
            const float x0 = x[e], x1 = x[e + 1];
            x[e] = fmaf(x0, cs, -x1 * sn);
            x[e + 1] = fmaf(x1, cs, x0 * sn);
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
    if (r >= heads) continue;
    if (is_q)
      reinterpret_cast<uint4*>(p.q_out + ((int64_t)t * p.hq + r) * D)[c] = w;
    else if (row0 >= 0)
      reinterpret_cast<uint4*>((is_v ? p.v_cache : p.k_cache) + row0 +
                               (int64_t)(r - nq - (is_v ? nk : 0)) * P * D)[c] = w;
  }
}

}  // namespace

hipError_t launch_rope_append(const RopeAppendParams& p, hipStream_t stream) {
  if (p.tokens == 0) return hipSuccess;
  // Up to a token per compute unit: every head of it at once (up to 64), for a short chain (1 token of 32
  // heads 3.9 -> 3.1 us, 64 tokens of 48 5.9 -> 4.3); more: small workgroups, which overlap better (2,600
  // tokens of 48 18.9 us, 29.1 with large ones).
  if (p.tokens <= 256)
    hipLaunchKernelGGL((rope_append_kernel<1024>), dim3(p.tokens), dim3(1024), 0, stream, p);
  else
    hipLaunchKernelGGL((rope_append_kernel<256>), dim3(p.tokens), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace qf
