// Position rotation of packed query and key heads, with an optional RMS norm of
// each head in the same pass:
//
//   x <- x / sqrt(mean(x^2) + eps) * weight   (qk_norm_rotary)
//   (a, b) of pair i -> (a cos - b sin, b cos + a sin) * mag,  angle = position * theta_i
//
// The angle is reduced in turns in float64 (position x turns per position, less its
// integer part) before the float32 sine and cosine: off by 2^-26 of a turn as it is rounded to
// float32, and by another 2^-24 at positions near 2^31, where 53 bits of turns per position end;
// in float32 a position of 10^5 would lose 2^-8 of a radian.
//
// HBM bound: every row is read and written once.  What a row's columns are multiplied
// with is formed once by its workgroup, into LDS, for all of its heads.  8192 rows of 40
// normed heads of 128, bf16 (168 MB): 38 us, 4.4 TB/s, where a copy of as many bytes
// runs at 4.8; 52 us with the norm weights in registers, the partner's columns loaded
// again and one head of a lane at a time.
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

// Heads with values above 2^59 or so, whose squares leave float32, are normed at 2^-70 of their size (an
// infinity or a NaN stays one); these are the only ones that cost more than a comparison.
constexpr float kTooLarge = 0x1p-70f;
__device__ __forceinline__ float inv_rms(float sum, int D, float eps) { return 1.0f / sqrtf(sum / (float)D + eps); }

// 8 columns as they are stored.
template <typename T>
struct Raw;
template <>
struct Raw<bf16_t> {
  uint4 u;
  __device__ __forceinline__ void load(const bf16_t* p) { u = *(const uint4*)p; }
  __device__ __forceinline__ void load(const bf16_t* p, const bf16_t* q) {  // 4 columns each
    const uint2 a = *(const uint2*)p, b = *(const uint2*)q;
    u = make_uint4(a.x, a.y, b.x, b.y);
  }
  __device__ __forceinline__ void get(float* f) const { unpack8(u, f); }
  __device__ __forceinline__ Raw across(int d) const {
    Raw r;
    r.u = make_uint4(__shfl_xor((int)u.x, d, 64), __shfl_xor((int)u.y, d, 64), __shfl_xor((int)u.z, d, 64),
                     __shfl_xor((int)u.w, d, 64));
    return r;
  }
};
template <>
struct Raw<float> {
  float v[8];
  __device__ __forceinline__ void load(const float* p) { load8(p, v); }
  __device__ __forceinline__ void load(const float* p, const float* q) {
    const float4 a = *(const float4*)p, b = *(const float4*)q;
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = v[e];
  }
  __device__ __forceinline__ Raw across(int d) const {
    Raw r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = __shfl_xor(v[e], d, 64);
    return r;
  }
};

// What each column of `rows` rows is multiplied with: y = (x A + partner B) / rms, with
// A = weight cos, B = -+ partner's weight sin (times mag; past the turning columns weight
// and 0), so that the norm weights cost a lane nothing.  With NORM a table each for the
// query and the key heads.  Column 8 c + e of D / 8 chunks stands at ((e / 2) chunks + c)
// float4 + e % 2 float2: lanes of consecutive chunks read consecutive 16 bytes.
template <bool NORM, bool INTER>
__device__ __forceinline__ void coefficients(const RotaryParams& p, int row0, int rows, float2* cs) {
  const int half = p.rd / 2, chunks = p.D / 8;
  const int tables = NORM && p.kv_heads > 0 ? 2 : 1;
  auto put = [&](int r, int t, int col, float a, float b) {
    cs[(r * tables + t) * p.D + (((col & 7) >> 1) * chunks + (col >> 3)) * 2 + (col & 1)] = make_float2(a, b);
  };
  for (int i = threadIdx.x; i < rows * half; i += kThreads) {
    const int r = i / half, k = i - r * half;
    const double turns = (double)p.pos[row0 + r] * p.theta[k];
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    s *= p.mag, c *= p.mag;
    const int e1 = INTER ? 2 * k : k, e2 = INTER ? 2 * k + 1 : k + half;
    for (int t = 0; t < tables; ++t) {
      const float* w = t ? p.wk : p.wq;
      const float w1 = NORM ? w[e1] : 1.0f, w2 = NORM ? w[e2] : 1.0f;
      put(r, t, e1, w1 * c, -w2 * s);
      put(r, t, e2, w2 * c, w1 * s);
    }
  }
  if constexpr (!NORM) {  // (the other columns are copied)
    __syncthreads();
    return;
  }
  const int rest = p.D - p.rd;
  for (int i = threadIdx.x; i < rows * rest; i += kThreads) {
    const int r = i / rest, col = p.rd + i - r * rest;
    for (int t = 0; t < tables; ++t) put(r, t, col, (t ? p.wk : p.wq)[col], 0.0f);
  }
  __syncthreads();
}

// LH lanes per head, 8 consecutive columns each (D <= 8 LH); RB rows per workgroup,
// hb heads per workgroup; U heads of a lane on their way together.  In the half
// layout a lane needs its partners' columns too: from the lane that has them where
// the whole head turns and fills its lanes (ACROSS), else read again, four at a time, as
// half of the turning columns need not be whole chunks (8192 rows of 32 normed heads of 48,
// 24 columns turning: 81 us column by column, 14 so).
template <typename T, int LH, bool NORM, bool INTER, bool ACROSS, int U>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryParams p, int RB, int hb) {
  extern __shared__ __align__(16) float2 cs[];
  constexpr int SLOTS = kThreads / LH;
  const int row0 = blockIdx.x * RB;
  const int rows = min(RB, p.M - row0);
  const int H = p.heads + p.kv_heads;
  const int h0 = blockIdx.y * hb, nh = min(hb, H - h0);
  const int slot = threadIdx.x / LH, c = threadIdx.x % LH;
  const int half = p.rd / 2, chunks = p.D / 8;
  const int tables = NORM && p.kv_heads > 0 ? 2 : 1;
  const int e0 = c * 8;
  const bool live = e0 < p.D;
  const bool turn = live && e0 < p.rd;                 // (whole chunks turn or stay)
  // half layout: the partners' first columns, of the first and of the last four
  const int pe0 = e0 >= half ? e0 - half : e0 + half, pe1 = e0 + 4 >= half ? e0 + 4 - half : e0 + 4 + half;
  const T* const x0 = (const T*)p.x + (int64_t)row0 * p.ldx + (int64_t)h0 * p.D;
  T* const y0 = (T*)p.y + (int64_t)row0 * p.ldy + (int64_t)h0 * p.D;
  // item it: row it / nh, head it % nh of this workgroup; a lane's first and its next
  const int items = rows * nh;
  int r = slot / nh, h = slot - r * nh;
  const int dr = SLOTS / nh, dh = SLOTS - dr * nh;
  Raw<T> v[U], o[U];
  int rr[U], hh[U];
  auto fetch = [&](int it) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      rr[u] = r, hh[u] = h;
      if (it + u * SLOTS < items) {
        const T* x = x0 + (int64_t)r * p.ldx + h * p.D;
        if (live) v[u].load(x + e0);
        if (!INTER && !ACROSS && turn) o[u].load(x + pe0, x + pe1);
      }
      r += dr, h += dh;
      if (h >= nh) h -= nh, ++r;
    }
  };
  fetch(slot);  // (the first heads are on their way while the coefficients are formed)
  coefficients<NORM, INTER>(p, row0, rows, cs);
  for (int it = slot; it < items; it += U * SLOTS) {
    float f[U][8], q[U][8];
    int fr[U], fh[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      v[u].get(f[u]);
      if constexpr (!INTER) (ACROSS ? v[u].across(LH / 2) : o[u]).get(q[u]);
      fr[u] = rr[u], fh[u] = hh[u];
    }
    fetch(it + U * SLOTS);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float inv = 1.0f;
      if constexpr (NORM) {
        auto squares = [&] {
          float sum = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(f[u][e], f[u][e], sum);
          sum = live ? sum : 0.0f;
#pragma unroll
          for (int d = LH / 2; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
          return sum;
        };
        const float sum = squares();
        inv = inv_rms(sum, p.D, p.eps);
        if (!(sum < INFINITY)) {  // (the same in all lanes of a head)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            f[u][e] *= kTooLarge;
            if constexpr (!INTER) q[u][e] *= kTooLarge;
          }
          inv = inv_rms(squares(), p.D, p.eps * (kTooLarge * kTooLarge));
        }
      }
      if (it + u * SLOTS >= items || !live) continue;
      T* const out = y0 + (int64_t)fr[u] * p.ldy + fh[u] * p.D + e0;
      if (!NORM && !turn) {
        store8(out, f[u]);
        continue;
      }
      const int t = tables == 2 && h0 + fh[u] >= p.heads ? 1 : 0;
      const float4* k = (const float4*)(cs + (fr[u] * tables + t) * p.D) + c;
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float4 ab = k[(e >> 1) * chunks];
        const float q0 = INTER ? f[u][e + 1] : q[u][e], q1 = INTER ? f[u][e] : q[u][e + 1];
        y[e] = turn ? __builtin_fmaf(q0, ab.y, f[u][e] * ab.x) : f[u][e] * ab.x;
        y[e + 1] = turn ? __builtin_fmaf(q1, ab.w, f[u][e + 1] * ab.z) : f[u][e + 1] * ab.z;
        if constexpr (NORM) y[e] *= inv, y[e + 1] *= inv;
      }
      store8(out, y);
    }
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
    float inv = 1.0f, size = 1.0f;
    if (p.wq) {
      auto squares = [&] {
        float sum = 0.0f;
        for (int e = lane; e < p.D; e += 64) {
          const float v = load1(x + e) * size;
          sum = __builtin_fmaf(v, v, sum);
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
        return sum;
      };
      const float sum = squares();
      inv = inv_rms(sum, p.D, p.eps);
      if (!(sum < INFINITY)) {
        size = kTooLarge;
        inv = inv_rms(squares(), p.D, p.eps * (kTooLarge * kTooLarge));
      }
    }
    const float* w = h >= p.heads ? p.wk : p.wq;
    for (int e = lane; e < p.D; e += 64) {
      float v = load1(x + e) * size;
      if (p.wq) v *= inv * w[e];
      if (e < p.rd) {
        const bool second = p.interleaved ? e & 1 : e >= half;
        const int pair = p.interleaved ? e >> 1 : (second ? e - half : e);
        const int pe = p.interleaved ? e ^ 1 : (second ? e - half : e + half);
        float o = load1(x + pe) * size;
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
  // Rows per workgroup: up to four share the latency of forming their coefficients while that leaves 1024
  // workgroups (8192 rows: 41 us alone, 38 by four, 40 by eight); few rows are spread over the heads instead.
  const int RB = std::min(4, std::max(1, p.M / 1024));
  int lh = 1;
  while (lh * 8 < p.D) lh *= 2;
  const bool fast = p.D % 8 == 0 && lh <= 64 && p.rd % 8 == 0 &&
                    (sizeof(T) == 2 || (p.ldx % 4 == 0 && p.ldy % 4 == 0));
  const int slots = fast ? kThreads / lh : kThreads / 64;
  const int hb = p.M >= 1024 ? H : std::min(H, slots);
  const dim3 grid((p.M + RB - 1) / RB, (H + hb - 1) / hb);
  if (!fast) {
    const size_t lds = (size_t)RB * half * sizeof(float2);
    rotary_any_kernel<T><<<grid, kThreads, lds, s>>>(p, RB, hb);
    return hipGetLastError();
  }
  const size_t lds = (size_t)RB * p.D * (p.wq && p.kv_heads > 0 ? 2 : 1) * sizeof(float2);
  const bool across = !p.interleaved && p.rd == p.D && p.D == 8 * lh && lh > 1;
#define BYOC_ROTARY_AS(LH, NORM, INTER, ACROSS) \
  rotary_kernel<T, LH, NORM, INTER, ACROSS, ACROSS ? 2 : 1><<<grid, kThreads, lds, s>>>(p, RB, hb)
#define BYOC_ROTARY(LH)                                                                      \
  case LH:                                                                                   \
    if (p.wq)                                                                                \
      p.interleaved ? BYOC_ROTARY_AS(LH, true, true, false)                                  \
                    : across ? BYOC_ROTARY_AS(LH, true, false, true) : BYOC_ROTARY_AS(LH, true, false, false);   \
    else                                                                                     \
      p.interleaved ? BYOC_ROTARY_AS(LH, false, true, false)                                 \
                    : across ? BYOC_ROTARY_AS(LH, false, false, true) : BYOC_ROTARY_AS(LH, false, false, false); \
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
#undef BYOC_ROTARY_AS
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& p, hipStream_t s) {
  if (p.D < 2 || p.D > 512 || p.rd < 2 || p.rd > p.D || p.rd % 2 != 0) return hipErrorInvalidValue;
  return p.f32 ? launch<float>(p, s) : launch<bf16_t>(p, s);
}

}  // namespace byoc
