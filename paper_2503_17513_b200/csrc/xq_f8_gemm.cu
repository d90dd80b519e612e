// Block-scaled E4M3 products of the 8-bit layer.
//   out[m][n] = bf16( sum over groups g of 2^(ex[m][g] + ew[n / 128][g]) * sum over k in g of qx[m][k] qw[n][k] )
// and the gated pair silu(G) * U of two such products.  Sums in fp32, one rounding at the end.
#include <cuda_bf16.h>

#include "xq_f8.h"
#include "xq_internal.h"
#include "xq_ptx.cuh"

using namespace xqptx;

namespace {

__device__ __forceinline__ float silu_mul(float g, float u) { return g / (1.f + expf(-g)) * u; }

// One CTA: 16 tokens x 128 channels, thread = one channel, K blocks through shared memory.
struct SimpleParams {
  const uint8_t *x, *sx;
  const uint8_t *w[2], *sw[2];
  __nv_bfloat16* out;
  uint8_t *out_codes, *out_scales;
  int M, N, Np, K, Kb;
};
constexpr int ST = 16;

template <bool GATED>
__global__ void __launch_bounds__(128) simple_kernel(const SimpleParams p) {
  __shared__ float xs[ST][128];
  __shared__ float red[4];
  const int t = threadIdx.x, n = blockIdx.x * 128 + t, m0 = blockIdx.y * ST, P = xq_f8_pitch(p.K);
  float acc[GATED ? 2 : 1][ST] = {};
  pdl_launch_dependents();
  pdl_wait();
  for (int kb = 0; kb < p.Kb; ++kb) {
    __syncthreads();
    for (int i = 0; i < ST; ++i) {
      const int m = m0 + i;
      float v = 0.f;
      if (m < p.M) v = ldexpf(xqf8::decode(p.x[(size_t)m * (p.Kb * 128) + kb * 128 + t]), (int)p.sx[(size_t)m * P + kb] - 127);
      xs[i][t] = v;
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < (GATED ? 2 : 1); ++h) {
      float s[ST] = {};
      for (int k = 0; k < 128; ++k) {
        const float w = xqf8::decode(p.w[h][xq_f8_code_offset(n, kb * 128 + k, p.Np)]);
#pragma unroll
        for (int i = 0; i < ST; ++i) s[i] = fmaf(w, xs[i][k], s[i]);
      }
      const int e = (int)p.sw[h][(size_t)blockIdx.x * P + kb] - 127;
#pragma unroll
      for (int i = 0; i < ST; ++i) acc[h][i] += ldexpf(s[i], e);
    }
  }
  for (int i = 0; i < ST; ++i) {
    const int m = m0 + i;
    if (m >= p.M) break;
    float v = GATED ? silu_mul(acc[0][i], acc[GATED ? 1 : 0][i]) : acc[0][i];
    if (!GATED || p.out) {
      if (n < p.N) p.out[(size_t)m * p.N + n] = __float2bfloat16_rn(v);
    } else {
      if (n >= p.N) v = 0.f;
      float a = fabsf(v);
      for (int o = 16; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
      __syncthreads();
      if ((t & 31) == 0) red[t >> 5] = a;
      __syncthreads();
      a = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
      const int b = xqf8::scale_byte(a);
      p.out_codes[(size_t)m * p.Np + n] = (uint8_t)xqf8::pack4(v * xqf8::inv_scale(b), 0.f, 0.f, 0.f);
      const int Po = xq_f8_pitch(p.N);
      if (t == 0) p.out_scales[(size_t)m * Po + blockIdx.x] = (uint8_t)b;
      if (blockIdx.x == 0 && t < Po - p.Np / 128) p.out_scales[(size_t)m * Po + p.Np / 128 + t] = 127;
    }
  }
}

template <bool GATED>
cudaError_t launch_simple(const uint8_t* codes, const uint8_t* scales, int M, const xq_f8_weights* w0, const xq_f8_weights* w1, void* out,
                          uint8_t* oc, uint8_t* os, cudaStream_t st) {
  SimpleParams p = {codes, scales, {w0->codes, w1->codes}, {w0->scales, w1->scales}, (__nv_bfloat16*)out, oc, os, M, w0->N, w0->Np, w0->K, w0->Kb};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(w0->Np / 128, (M + ST - 1) / ST);
  cfg.blockDim = dim3(128);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, simple_kernel<GATED>, p);
}

}  // namespace

cudaError_t xq_f8_launch_gemm(const uint8_t* codes, const uint8_t* scales, int32_t M, const xq_f8_weights* w, void* out,
                              int32_t* status, cudaStream_t st) {
  (void)status;
  return launch_simple<false>(codes, scales, M, w, w, out, nullptr, nullptr, st);
}

cudaError_t xq_f8_launch_gated(const uint8_t* codes, const uint8_t* scales, int32_t M, const xq_f8_weights* gate,
                               const xq_f8_weights* up, void* out, uint8_t* out_codes, uint8_t* out_scales, int32_t* status,
                               cudaStream_t st) {
  (void)status;
  return launch_simple<true>(codes, scales, M, gate, up, out, out_codes, out_scales, st);
}
