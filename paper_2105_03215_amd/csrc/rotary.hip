// Position rotation of packed query and key heads, with an optional RMS norm of
// each head in the same pass:
//
//   x <- x / sqrt(mean(x^2) + eps) * weight   (qk_norm_rotary)
//   (a, b) of pair i -> (a cos - b sin, b cos + a sin) * mag,  angle = position * theta_i
//
// The angle is reduced in turns in float64 (position x turns per position, less its
// integer part), exact enough for every 32-bit position, before the float32 sine
// and cosine; in float32 a position of 10^5 would lose 2^-8 of a radian.
//
// HBM bound: every row is read and written once.  A row's angles are formed once by
// its workgroup, into LDS, for all of its heads.
#include <algorithm>

#include "device_common.h"

namespace byoc {
namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* v) {
  if constexpr (sizeof(T) == 2) {
    unpack8(*(const uint4*)p, v);
  } else {
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* v) {
  if constexpr (sizeof(T) == 2) {
    *(uint4*)p = pack8(v);
  } else {
    *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
    *(float4*)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
}

__device__ __forceinline__ float load1(const bf16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { *p = f32_to_bf16(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

// cos and sin (times mag) of the pairs of `rows` rows from row0 on, into cs[row][pair]
__device__ __forceinline__ void angles(const RotaryParams& p, int row0, int rows, float2* cs) {
  const int half = p.rd / 2;
  for (int i = threadIdx.x; i < rows * half; i += kThreads) {
    const int r = i / half;
    const double turns = (double)p.pos[row0 + r] * p.theta[i - r * half];
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    cs[i] = make_float2(c * p.mag, s * p.mag);
  }
  __syncthreads();
}

// LH lanes per head, 8 consecutive columns each (D <= 8 LH); RB rows per workgroup,
// hb heads per workgroup.
template <typename T, int LH, bool NORM, bool INTER>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryParams p, int RB, int hb) {
  extern __shared__ float2 cs[];
  constexpr int SLOTS = kThreads / LH;
  const int row0 = blockIdx.x * RB;
  const int rows = min(RB, p.M - row0);
  angles(p, row0, rows, cs);
  const int H = p.heads + p.kv_heads;
  const int h0 = blockIdx.y * hb, nh = min(hb, H - h0);
  const int slot = threadIdx.x / LH, c = threadIdx.x % LH;
  const int half = p.rd / 2;
  const int e0 = c * 8;
  const bool live = e0 < p.D;
  // columns of this lane that turn, and in the half layout its partner's
  const bool turn = live && e0 < p.rd;
  const bool second = !INTER && e0 >= half;
  const int pe = second ? e0 - half : e0 + half;  // the partner's first column
  const int pair = INTER ? e0 / 2 : (second ? e0 - half : e0);
  float w[2][8], pw[2][8];
  if constexpr (NORM) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float* g = k == 0 ? p.wq : (p.wk ? p.wk : p.wq);
      if (live) load8(g + e0, w[k]);
      if (!INTER && turn) load8(g + pe, pw[k]);
    }
  }
  for (int it = slot; it < rows * nh; it += SLOTS) {
    const int r = it / nh, h = h0 + it - r * nh;
    const T* x = (const T*)p.x + (int64_t)(row0 + r) * p.ldx + (int64_t)h * p.D;
    T* y = (T*)p.y + (int64_t)(row0 + r) * p.ldy + (int64_t)h * p.D;
    float v[8], o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = o[e] = 0.0f;
    if (live) load8(x + e0, v);
    if (!INTER && turn) load8(x + pe, o);
    if constexpr (NORM) {
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(v[e], v[e], sum);
#pragma unroll
      for (int d = LH / 2; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
      const float inv = 1.0f / sqrtf(sum / (float)p.D + p.eps);
      const bool key = h >= p.heads;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] *= inv * (key ? w[1][e] : w[0][e]);
        if (!INTER) o[e] *= inv * (key ? pw[1][e] : pw[0][e]);
      }
    }
    if (turn) {
      const float2* t = cs + r * half + pair;
      if constexpr (INTER) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float a = v[2 * e], b = v[2 * e + 1];
          v[2 * e] = a * t[e].x - b * t[e].y;
          v[2 * e + 1] = b * t[e].x + a * t[e].y;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = v[e] * t[e].x + (second ? o[e] : -o[e]) * t[e].y;
      }
    }
    if (live) store8(y + e0, v);
  }
}

// Any head size, pair layout and alignment: a wave per (row, head), one column
// per lane at a time.
template <typename T>
__global__ __launch_bounds__(kThreads) void rotary_any_kernel(RotaryParams p, int RB, int hb) {
  extern __shared__ float2 cs[];
  const int row0 = blockIdx.x * RB;
  const int rows = min(RB, p.M - row0);
  angles(p, row0, rows, cs);
  const int H = p.heads + p.kv_heads;
  const int h0 = blockIdx.y * hb, nh = min(hb, H - h0);
  const int half = p.rd / 2;
  const int lane = threadIdx.x & 63;
  for (int it = threadIdx.x >> 6; it < rows * nh; it += kThreads / 64) {
    const int r = it / nh, h = h0 + it - r * nh;
    const T* x = (const T*)p.x + (int64_t)(row0 + r) * p.ldx + (int64_t)h * p.D;
    T* y = (T*)p.y + (int64_t)(row0 + r) * p.ldy + (int64_t)h * p.D;
    float inv = 1.0f;
    if (p.wq) {
      float sum = 0.0f;
      for (int e = lane; e < p.D; e += 64) {
        const float v = load1(x + e);
        sum = __builtin_fmaf(v, v, sum);
      }
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
      inv = 1.0f / sqrtf(sum / (float)p.D + p.eps);
    }
    const float* w = h >= p.heads ? p.wk : p.wq;
    for (int e = lane; e < p.D; e += 64) {
      float v = load1(x + e);
      if (p.wq) v *= inv * w[e];
      if (e < p.rd) {
        const bool second = p.interleaved ? e & 1 : e >= half;
        const int pair = p.interleaved ? e >> 1 : (second ? e - half : e);
        const int pe = p.interleaved ? e ^ 1 : (second ? e - half : e + half);
        float o = load1(x + pe);
        if (p.wq) o *= inv * w[pe];
        const float2 t = cs[r * half + pair];
        v = v * t.x + (second ? o : -o) * t.y;
      }
      store1(y + e, v);
    }
  }
  // the padding columns of a bf16 row are zero
  if (blockIdx.y == 0)
    for (int r = threadIdx.x; r < rows; r += kThreads)
      for (int c = H * p.D; c < p.cols_out; ++c) store1((T*)p.y + (int64_t)(row0 + r) * p.ldy + c, 0.0f);
}

template <typename T>
hipError_t launch(const RotaryParams& p, hipStream_t s) {
  const int H = p.heads + p.kv_heads;
  const int half = p.rd / 2;
  // Rows per workgroup: four share the angles' latency once there are enough of them for the chip;
  // few rows are spread over the heads instead.
  const int RB = p.M >= 2048 ? 4 : 1;
  int lh = 1;
  while (lh * 8 < p.D) lh *= 2;
  const bool fast = p.D % 8 == 0 && lh <= 64 && (p.interleaved ? p.rd : half) % 8 == 0 &&
                    (sizeof(T) == 2 || (p.ldx % 4 == 0 && p.ldy % 4 == 0));
  const int slots = fast ? kThreads / lh : kThreads / 64;
  const int hb = p.M >= 1024 ? H : std::min(H, slots);
  const dim3 grid((p.M + RB - 1) / RB, (H + hb - 1) / hb);
  const size_t lds = (size_t)RB * half * sizeof(float2);
  if (!fast) {
    rotary_any_kernel<T><<<grid, kThreads, lds, s>>>(p, RB, hb);
    return hipGetLastError();
  }
#define BYOC_ROTARY(LH)                                                                              \
  case LH:                                                                                           \
    if (p.wq)                                                                                        \
      p.interleaved ? rotary_kernel<T, LH, true, true><<<grid, kThreads, lds, s>>>(p, RB, hb)        \
                    : rotary_kernel<T, LH, true, false><<<grid, kThreads, lds, s>>>(p, RB, hb);      \
    else                                                                                             \
      p.interleaved ? rotary_kernel<T, LH, false, true><<<grid, kThreads, lds, s>>>(p, RB, hb)       \
                    : rotary_kernel<T, LH, false, false><<<grid, kThreads, lds, s>>>(p, RB, hb);     \
    break;
  switch (lh) {
    BYOC_ROTARY(1)
    BYOC_ROTARY(2)
    BYOC_ROTARY(4)
    BYOC_ROTARY(8)
    BYOC_ROTARY(16)
    BYOC_ROTARY(32)
    BYOC_ROTARY(64)
  }
#undef BYOC_ROTARY
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& p, hipStream_t s) {
  if (p.D < 2 || p.D > 512 || p.rd < 2 || p.rd > p.D || p.rd % 2 != 0) return hipErrorInvalidValue;
  return p.f32 ? launch<float>(p, s) : launch<bf16_t>(p, s);
}

}  // namespace byoc
