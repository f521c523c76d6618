// The gated feed-forward block in fp32 for any width, stride and alignment (formulas, and the kernels for multiples of four: glu_ffn.hip).  The products are the fp32 matrix-core products of the framework's MLPs; the
// gate between them is one pass over [g, u], bound by memory.  exp and erf are the full-precision ones: nothing here is rounded to fewer bits (1 + erf is within 6e-8, not of itself).
#include <algorithm>
#include "kernels.h"
#include "token_ops.h"

namespace sama {
namespace {

template <int ACT>
__device__ __forceinline__ void gate_and_slope32(float g, float& a, float& da) {
  if constexpr (ACT == GLU_GELU) {
    const float cdf = 0.5f * (1.f + erff(g * 0.70710678118654752f));
    a = g * cdf; da = fmaf(g * 0.39894228040143268f, expf(-0.5f * g * g), cdf);
  } else {
    const float s = 1.f / (1.f + expf(-g));
    a = g * s; da = fmaf(a, 1.f - s, s);
  }
}

// pre [T x 2F] = [g, u].  BACKWARD: dpre = [dh u act'(g), dh act(g)], else h = act(g) u [T x F]
template <int ACT, bool BACKWARD>
__global__ __launch_bounds__(256) void k_gate_f32(const float* __restrict__ pre, const float* __restrict__ dh, float* __restrict__ out, int64_t T, int F) {
  for (int64_t t = blockIdx.y; t < T; t += gridDim.y) {
    const float *g = pre + t * 2 * F, *u = g + F;
    for (int f = blockIdx.x * 256 + threadIdx.x; f < F; f += gridDim.x * 256) {
      float a, da;
      gate_and_slope32<ACT>(g[f], a, da);
      if constexpr (BACKWARD) {
        const float d = dh[t * F + f];
        out[t * 2 * F + f] = d * (u[f] * da);
        out[t * 2 * F + F + f] = d * a;
      } else {
        out[t * F + f] = a * u[f];
      }
    }
  }
}
template <bool BACKWARD>
void launch_gate(hipStream_t st, int act, const float* pre, const float* dh, float* out, int64_t T, int F) {
  ProfScope ps(st, F_OTHER, (BACKWARD ? 20.0 : 12.0) * T * F);
  const dim3 grid((F + 255) / 256, (uint32_t)std::min<int64_t>(T, 65535));
  if (act == GLU_GELU) launch_kernel(ps, k_gate_f32<GLU_GELU, BACKWARD>, grid, 256, 0, st, pre, dh, out, T, F);
  else launch_kernel(ps, k_gate_f32<GLU_SILU, BACKWARD>, grid, 256, 0, st, pre, dh, out, T, F);
}
size_t up256(size_t b) { return (b + 255) / 256 * 256; }
GemmF32Args product(const void* A, int64_t sa_i, int64_t sa_k, const void* B, int64_t sb_k, int64_t sb_j, void* C, int64_t ldc, int M, int N, int K) {
  GemmF32Args g{};
  g.A = (const float*)A; g.sa_i = sa_i; g.sa_k = sa_k; g.B = (const float*)B; g.sb_k = sb_k; g.sb_j = sb_j;
  g.C = (float*)C; g.ldc = ldc; g.M = M; g.N = N; g.K = K;
  return g;
}
}  // namespace

size_t glu_ffn_plain_bytes(int64_t T, int F) { return up256((size_t)T * 2 * F * 4); }
size_t glu_ffn_plain_grad_bytes(int64_t T, int F) { return up256((size_t)T * F * 4) + up256((size_t)T * 2 * F * 4); }

void launch_glu_ffn_plain(hipStream_t st, const GluFfnArgs& a, void* workspace) {
  const int T = (int)a.T, d = a.d, F = a.F;
  float* const pre = (float*)(a.saved != nullptr ? a.saved : workspace);
  const GemmF32Args up = product(a.x, a.ldx, 1, a.w_in, 1, d, pre, 2 * (int64_t)F, T, 2 * F, d);
  launch_gemm_f32_batch(st, &up, 1);
  launch_gate<false>(st, a.act, pre, nullptr, (float*)a.hidden, T, F);
  const GemmF32Args down = product(a.hidden, F, 1, a.w_out, 1, F, a.y, a.ldy, T, d, F);
  launch_gemm_f32_batch(st, &down, 1);
}

void launch_glu_ffn_grad_plain(hipStream_t st, const GluFfnGradArgs& a, void* workspace) {
  const int T = (int)a.T, d = a.d, F = a.F;
  float* const dh = (float*)workspace;
  float* const dpre = (float*)((char*)workspace + up256((size_t)T * F * 4));
  const GemmF32Args first[2] = {product(a.dy, a.lddy, 1, a.w_out, F, 1, dh, F, T, F, d),
                                product(a.dy, 1, a.lddy, a.hidden, F, 1, a.dw_out, F, d, F, T)};
  launch_gemm_f32_batch(st, first, 2);
  launch_gate<true>(st, a.act, (const float*)a.saved, dh, dpre, T, F);
  const GemmF32Args second[2] = {product(dpre, 2 * (int64_t)F, 1, a.w_in, d, 1, a.dx, a.lddx, T, d, 2 * F),
                                 product(dpre, 1, 2 * (int64_t)F, a.x, a.ldx, 1, a.dw_in, d, 2 * F, d, T)};
  launch_gemm_f32_batch(st, second, 2);
}

}  // namespace sama
