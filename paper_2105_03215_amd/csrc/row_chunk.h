// Rows of any width, 8 values at a time.
#pragma once

#include "device_common.h"

namespace byoc {

// 8 consecutive values of a row as they are stored, zero from column K on.  Rows are
// any number of columns apart, so that they need only be aligned to a value: the
// memory takes 16 bytes at any address (8000 x 513 x 3001, bf16: 83 us value by
// value, 49 so).
struct __attribute__((packed, aligned(4))) F32x4u {
  float v[4];
};
struct __attribute__((packed, aligned(2))) Bf16x8u {
  uint32_t v[4];
};
template <bool F32>
struct Chunk;
template <>
struct Chunk<true> {
  float v[8];
  __device__ __forceinline__ void load(const void* x, int64_t row, int col, int K) {
    const float* p = (const float*)x + row + col;
    if (col + 8 <= K) {
      const F32x4u a = *(const F32x4u*)p, b = *(const F32x4u*)(p + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = a.v[e], v[4 + e] = b.v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = col + e < K ? p[e] : 0.0f;
    }
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = v[e];
  }
};
template <>
struct Chunk<false> {
  uint4 u;
  __device__ __forceinline__ void load(const void* x, int64_t row, int col, int K) {
    const bf16_t* p = (const bf16_t*)x + row + col;
    if (col + 8 <= K) {
      const Bf16x8u a = *(const Bf16x8u*)p;
      u = make_uint4(a.v[0], a.v[1], a.v[2], a.v[3]);
    } else {
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = col + e < K ? p[e] : 0u;
      u = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    }
  }
  __device__ __forceinline__ void get(float* f) const { unpack8(u, f); }
};

// The same of a row that is written: the columns below `end`.
template <bool F32>
__device__ __forceinline__ void store_chunk(void* y, int64_t row, int col, int end, const float* v) {
  if constexpr (F32) {
    float* p = (float*)y + row + col;
    if (col + 8 <= end) {
      *(F32x4u*)p = F32x4u{v[0], v[1], v[2], v[3]};
      *(F32x4u*)(p + 4) = F32x4u{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < end) p[e] = v[e];
    }
  } else {
    bf16_t* p = (bf16_t*)y + row + col;
    if (col + 8 <= end) {
      const uint4 u = pack8(v);
      *(Bf16x8u*)p = Bf16x8u{u.x, u.y, u.z, u.w};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < end) p[e] = f32_to_bf16(v[e]);
    }
  }
}

}  // namespace byoc
