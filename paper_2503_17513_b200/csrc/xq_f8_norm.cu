// Residual addition, RMS norm and quantization to E4M3 in one pass over a token row:
//   t = x + r;  sum = bf16(t);  y = t / sqrt(mean(t^2) + eps) * gamma;  codes, scales = Q(y)
// with everything between the bf16 inputs and the outputs in fp32: t is not rounded before the norm (the bf16 sum is an
// output, not an intermediate), and y is rounded once, to 8 bits (and once to bf16 where the caller wants it too).
//
// Bound by HBM: 2 + 2 bytes in, 2 + 1 bytes out per element.  A row lives in the registers of one CTA between the two
// reductions, so that every byte crosses once.  Thread t holds vectors t, t + T, ... of eight channels (16-byte loads); the
// 128 channels of a group are the vectors of one half-warp, so that the group's maximum is four shuffles.
#include <cuda_bf16.h>

#include "xq_f8.h"
#include "xq_internal.h"
#include "xq_ptx.cuh"

using namespace xqptx;

namespace {

struct Vec8 {
  float v[8];
};

// eight bf16 from p, the first n of them inside the row (n >= 8: one 16-byte load)
__device__ __forceinline__ Vec8 load8(const __nv_bfloat16* p, int n) {
  Vec8 r;
  if (n >= 8) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.v[2 * i] = __uint_as_float(w[i] << 16);
      r.v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = i < n ? __bfloat162float(p[i]) : 0.f;
  }
  return r;
}

__device__ __forceinline__ void store8(__nv_bfloat16* p, const Vec8& r, int n) {
  if (n >= 8) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(r.v[2 * i], r.v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = __float2bfloat16_rn(r.v[i]);
  }
}

template <int V>
__global__ void __launch_bounds__(1024) norm_quant_kernel(const XqF8NormArgs a) {
  __shared__ float part[2][32];
  const int t = threadIdx.x, T = blockDim.x, lane = t & 31, warp = t >> 5;
  const int Kq = xq_f8_padded(a.K), P = xq_f8_pitch(a.K);
  pdl_launch_dependents();
  pdl_wait();
  int flip = 0;
  for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x, flip ^= 1) {
    const __nv_bfloat16* x = (const __nv_bfloat16*)a.x + m * a.ldx;
    const __nv_bfloat16* r = a.residual ? (const __nv_bfloat16*)a.residual + m * a.ldr : nullptr;
    Vec8 v[V];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = 8 * (t + i * T), n = a.K - c;
      if (n > 0) {
        v[i] = load8(x + c, n);
        if (r) {
          const Vec8 w = load8(r + c, n);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i].v[j] += w.v[j];
        }
        if (a.sum) store8((__nv_bfloat16*)a.sum + m * a.ldr + c, v[i], n);
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(v[i].v[j], v[i].v[j], ss);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i].v[j] = 0.f;
      }
    }
    float rstd = 1.f;
    if (a.gamma) {
      for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      // two sets of partial sums in turn: a row's are still being read when the next row's first ones arrive
      if (lane == 0) part[flip][warp] = ss;
      __syncthreads();
      ss = lane < (T >> 5) ? part[flip][lane] : 0.f;
      for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      rstd = 1.f / sqrtf(ss / (float)a.K + a.eps);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = 8 * (t + i * T), n = a.K - c;
      if (a.gamma && n > 0) {
        const Vec8 g = load8((const __nv_bfloat16*)a.gamma + c, n);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i].v[j] = v[i].v[j] * rstd * g.v[j];
        if (a.y) store8((__nv_bfloat16*)a.y + m * a.ldy + c, v[i], n);
      }
      float amax = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(v[i].v[j]));
      for (int o = 8; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      if (c < Kq) {
        const int b = xqf8::scale_byte(amax);
        const float s = xqf8::inv_scale(b);
        uint2 q;
        q.x = xqf8::pack4(v[i].v[0] * s, v[i].v[1] * s, v[i].v[2] * s, v[i].v[3] * s);
        q.y = xqf8::pack4(v[i].v[4] * s, v[i].v[5] * s, v[i].v[6] * s, v[i].v[7] * s);
        *reinterpret_cast<uint2*>(a.codes + m * (int64_t)Kq + c) = q;
        if ((lane & 15) == 0) a.scales[m * (int64_t)P + (c >> 7)] = (uint8_t)b;
      }
    }
    if (t < P - Kq / 128) a.scales[m * (int64_t)P + Kq / 128 + t] = 127;
  }
}

template <int V>
cudaError_t launch(const XqF8NormArgs& a, int sms, cudaStream_t st) {
  const int vecs = xq_f8_padded(a.K) / 8;
  const int T = ((vecs + V - 1) / V + 31) / 32 * 32;
  const int resident = 2048 / T > 0 ? 2048 / T : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.M < sms * resident ? a.M : sms * resident));
  cfg.blockDim = dim3(T);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, norm_quant_kernel<V>, a);
}

}  // namespace

cudaError_t xq_f8_launch_norm_quant(const XqF8NormArgs& a, int sms, cudaStream_t st) {
  const int vecs = xq_f8_padded(a.K) / 8;
  if (vecs <= 1024) return launch<1>(a, sms, st);
  if (vecs <= 2048) return launch<2>(a, sms, st);
  if (vecs <= 4096) return launch<4>(a, sms, st);
  return launch<8>(a, sms, st);
}
