// What the dense products on codes (8-bit and microscaled 4-bit) share at their end.
#pragma once

#include "row_chunk.h"

namespace byoc {

// GELU for bf16 outputs: gelu's polynomial with exp(-a^2) straight from the hardware's
// exp2, without the residual of the square: 18 instructions in place of 29, relative
// error below 2^-18 down to x = -5 and 2^-16 to -9, where the output's rounding is 2^-8
// (1024 x 768 x 3072, quantization included: 15.3 us with gelu, 13.9 with this).
__device__ __forceinline__ float gelu_short(float v) {
  constexpr float kErfcP[9] = {2.820777595e-01f, 2.825488448e-01f, 2.416709065e-01f, 2.090727836e-01f,
                               -4.348613694e-02f, 3.051838875e-01f, -5.132555962e-01f, 2.983081341e-01f,
                               -6.212075427e-02f};
  const float a = fminf(fabsf(v) * 0.70710678118654752440f, 10.0f);
  const float k = __builtin_amdgcn_rcpf(__builtin_fmaf(0.5f, a, 1.0f));
  float p = kErfcP[8];
#pragma unroll
  for (int i = 7; i >= 0; --i) p = __builtin_fmaf(p, k, kErfcP[i]);
  const float e = __builtin_amdgcn_exp2f(a * -1.44269504088896340736f * a);
  const float half = 0.5f * k * p * e;  // erfc(a) / 2
  return v * (v < 0.0f ? half : 1.0f - half);
}

// The activation, which keeps a NaN (the row of an infinity or a NaN; the clamp's
// median would drop it).
template <bool F32, int MODE>
__device__ __forceinline__ float act_nan(float v, ActClamp ac) {
  if constexpr (MODE == 1) return F32 ? gelu(v) : gelu_short(v);
  const float y = act_apply<MODE>(v, ac);
  return v != v ? v : y;
}

__device__ __forceinline__ void load8f(const float* p, float* v) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

// Eight columns of a row of the residual (zeros without one).
template <bool F32, class P>
__device__ __forceinline__ Chunk<F32> load_res(const P& p, int64_t m, int n) {
  Chunk<F32> r;
  if constexpr (F32) {
    r.load(p.res, m * p.ldr, n, p.res ? p.N : 0);
  } else {
    r.load(p.res, m * p.ldr, n, p.res ? (p.ldr % 8 == 0 ? (int)p.ldr : p.channels) : 0);
  }
  return r;
}

}  // namespace byoc
