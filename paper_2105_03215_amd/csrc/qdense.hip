// Dense composite on 8-bit codes with a scale for each token and each output
// channel: the rows of the activations are quantized on the way in (quant_rows),
// multiplied on int8 MFMA with exact int32 sums, and rescaled in the epilogue.
//
//   a_m = max_k |x_mk|,  q_mk = rint(127 x_mk / a_m),
//   y_mn = act((sum_k q_mk r_nk) (a_m / 127) (b_n / 127) + bias_n + res_mn)
//
// with r, b the same of the weight rows, formed once at engine creation by the
// same kernel.
#include <type_traits>

#include "lds_dma.h"

namespace byoc {
namespace {

using namespace dma;

// 8 consecutive values of a row, zero from column K on.  f32 rows need not be
// 16-byte aligned (their stride is any number of columns); bf16 rows are, but for
// constants of other widths (`vec` false).
struct __attribute__((packed, aligned(4))) F32x4u {
  float v[4];
};
template <bool F32>
__device__ __forceinline__ void load8(const void* x, int64_t row, int col, int K, bool vec, float* v) {
  if constexpr (F32) {
    const float* p = (const float*)x + row + col;
    if (col + 8 <= K) {
      const F32x4u a = *(const F32x4u*)p, b = *(const F32x4u*)(p + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = a.v[e], v[4 + e] = b.v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = col + e < K ? p[e] : 0.0f;
    }
  } else {
    if (!vec) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = col + e < K ? bf16_to_f32(((const bf16_t*)x)[row + col + e]) : 0.0f;
    } else if (col < K) {
      unpack8(*(const uint4*)((const bf16_t*)x + row + col), v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = col + e < K ? v[e] : 0.0f;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    }
  }
}

// A row's scale, and what its codes are formed with.  The magnitudes are compared
// as integers, which orders NaN above infinity above every number.
struct RowScale {
  float scale;  // a / 127, NaN when the row holds an infinity or a NaN
  float pre;    // power of two that keeps 127 x and 1 / a in range
  float a, inv;
  bool codes;   // false: all codes are zero
};
__device__ __forceinline__ RowScale row_scale(uint32_t bits) {
  RowScale r;
  const float a = __uint_as_float(bits);
  const bool finite = bits < 0x7F800000u;
  r.codes = finite && bits != 0u;
  r.scale = finite ? a / 127.0f : __uint_as_float(0x7FC00000u);
  r.pre = a < 0x1p-60f ? 0x1p64f : (a > 0x1p60f ? 0x1p-64f : 1.0f);
  r.a = a * r.pre;
  r.inv = __builtin_amdgcn_rcpf(r.a);
  return r;
}
// rint(127 x / a): the quotient rounded to float32 first, as a correctly rounded
// division gives it (a bf16 quotient that is not half-way between two codes is at least
// 2^-10 away from it, so that for bf16 values the code is that of the exact quotient)
template <bool F32>
__device__ __forceinline__ float code_of(float x, const RowScale& r) {
  const float n = 127.0f * (x * r.pre);
  float y;
  if constexpr (F32) {
    y = n / r.a;
  } else {
    y = n * r.inv;
    y = __builtin_fmaf(__builtin_fmaf(-y, r.a, n), r.inv, y);
  }
  return r.codes ? __builtin_rintf(y) : 0.0f;
}
__device__ __forceinline__ uint32_t pack_codes(const float* y) {
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) w = put_u8(y[e] + 128.0f, e, w);
  return w ^ kU8ToCode;
}

// WPR waves per row; NC > 0: the row's chunks of 8 stay in registers between the
// maximum and the codes (at most NC per lane), NC = 0: they are read twice.
template <bool F32, int WPR, int NC>
__global__ __launch_bounds__(256) void quant_rows_kernel(QRowsParams p) {
  constexpr int LANES = 64 * WPR;
  __shared__ uint32_t tops[4];
  const int tid = threadIdx.x, wave = tid >> 6;
  const int row = blockIdx.x * (4 / WPR) + tid / LANES;
  const int lane = tid % LANES;
  const int chunks = p.Kq / 8;
  const bool live = row < p.M, vec = p.ldx % 8 == 0;
  const int64_t at = (int64_t)row * p.ldx;
  uint32_t top = 0;
  float v[NC > 0 ? NC : 1][8];
  auto widen = [&](const float* f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7FFFFFFFu);
  };
  if constexpr (NC > 0) {
#pragma unroll
    for (int i = 0; i < NC; ++i) load8<F32>(p.x, at, (i * LANES + lane) * 8, live ? p.K : 0, vec, v[i]);
#pragma unroll
    for (int i = 0; i < NC; ++i) widen(v[i]);
  } else {
    for (int c = lane; c < chunks; c += LANES) {
      load8<F32>(p.x, at, c * 8, live ? p.K : 0, vec, v[0]);
      widen(v[0]);
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
  if constexpr (WPR == 4) {
    if ((tid & 63) == 0) tops[wave] = top;
    __syncthreads();
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  }
  if (row >= p.rows) return;
  const RowScale r = row_scale(top);
  if (lane == 0) p.scale[row] = r.scale;
  int8_t* q = p.q + (int64_t)row * p.Kq;
  auto write = [&](int c, const float* f) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = code_of<F32>(f[e], r);
    *(uint2*)(q + c * 8) = make_uint2(pack_codes(y), pack_codes(y + 4));
  };
  if constexpr (NC > 0) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int c = i * LANES + lane;
      if (c < chunks) write(c, v[i]);
    }
  } else {
    for (int c = lane; c < chunks; c += LANES) {
      load8<F32>(p.x, at, c * 8, live ? p.K : 0, vec, v[0]);
      write(c, v[0]);
    }
  }
}

template <bool F32>
void quant_rows(const QRowsParams& p, hipStream_t s) {
  const int rows4 = (p.rows + 3) / 4;
  const int c = p.Kq / 8;  // chunks of a row
  if (c <= 64) quant_rows_kernel<F32, 1, 1><<<rows4, 256, 0, s>>>(p);
  else if (c <= 128) quant_rows_kernel<F32, 1, 2><<<rows4, 256, 0, s>>>(p);
  else if (c <= 512) quant_rows_kernel<F32, 4, 2><<<p.rows, 256, 0, s>>>(p);
  else if (c <= 1024) quant_rows_kernel<F32, 4, 4><<<p.rows, 256, 0, s>>>(p);
  else quant_rows_kernel<F32, 4, 0><<<p.rows, 256, 0, s>>>(p);
}

constexpr int kCH = 8;   // 16-byte chunks of an LDS row
constexpr int kBK = 128;  // codes of a stage

__device__ __forceinline__ i32x4 mma(uint4 a, uint4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// The activation, which keeps a NaN (the row of an infinity or a NaN; the clamp's
// median would drop it).
template <int MODE>
__device__ __forceinline__ float act_nan(float v, ActClamp ac) {
  const float y = act_apply<MODE>(v, ac);
  return MODE != 1 && v != v ? v : y;
}

// Eight columns of one output row: y = act(acc * scale + bias + res).
template <bool F32, int MODE>
__device__ __forceinline__ void finish8(const QDenseParams& p, const int* acc, float xs, const float* ws,
                                        const float* bias, int64_t m, int n, ActClamp ac) {
  float r[8], v[8];
  if constexpr (F32) {
    const float* rp = (const float*)p.res + m * p.ldr + n;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = p.res && n + e < p.N ? rp[e] : 0.0f;
  } else {
    unpack8(p.res ? *(const uint4*)((const bf16_t*)p.res + m * p.ldr + n) : make_uint4(0u, 0u, 0u, 0u), r);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = act_nan<MODE>(__builtin_fmaf((float)acc[e], xs * ws[e], bias[e]) + r[e], ac);
  if constexpr (F32) {
    float* y = (float*)p.y + m * p.ldy + n;
    if (p.ldy % 4 == 0 && n + 8 <= p.N) {
      *(float4*)y = make_float4(v[0], v[1], v[2], v[3]);
      *(float4*)(y + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (n + e < p.N) y[e] = v[e];
    }
  } else {
    *(uint4*)((bf16_t*)p.y + m * p.ldy + n) = pack8(v);
  }
}

__device__ __forceinline__ void load8f(const float* p, float* v) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

// BM rows x BN channels per workgroup of WM x WN waves; both operands streamed
// HBM -> LDS in stages of 128 codes through a ring of NS, the MFMA operands of a
// step of 64 codes read while the previous step multiplies.
template <int BM, int BN, int WM, int WN, int NS, bool F32>
__global__ __launch_bounds__(64 * WM * WN) void qdense_kernel(QDenseParams p) {
  constexpr int kNT = 64 * WM * WN;
  constexpr int kRowsPerPass = kNT / kCH;
  constexpr int WTM = BM / WM, WTN = BN / WN;
  constexpr int TM = WTM / 16, TN = WTN / 16;
  constexpr int AR = BM / kRowsPerPass, BR = BN / kRowsPerPass;
  static_assert(BM % kRowsPerPass == 0 && BN % kRowsPerPass == 0 && kRowsPerPass % 16 == 0, "fill shape");
  static_assert(WTM % 16 == 0 && WTN % 32 == 0, "wave tile: whole MFMA rows, pairs of channel tiles");
  constexpr int LPS = AR + BR;
  constexpr int STAGE = (BM + BN) * kCH;  // uint4 per stage
  static_assert(NS >= 2 && (NS - 1) * LPS <= 63, "vmcnt immediate");
  static_assert(NS * STAGE * 16 <= kLdsLimit, "LDS");
  __shared__ uint4 ring[NS * STAGE];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int r0 = tid / kCH;
  const int cva = (lane & 7) ^ (r0 & 7);
  const int cvb = (lane & 7) ^ ((r0 & 3) | ((r0 & 8) >> 1));

  // XCD x = (gx, gy) of 8 / py x py owns a block of the tile grid (workgroup b runs on XCD b % 8)
  const int ntm = (p.M + BM - 1) / BM, ntn = (p.N + BN - 1) / BN;
  const int x = blockIdx.x & 7, j = blockIdx.x >> 3;
  const int px = 8 / p.py;
  const int mh = (ntm + px - 1) / px, nh = (ntn + p.py - 1) / p.py;
  const int gx = x / p.py, gy = x - gx * p.py;
  const int jm = j / nh;
  const int tm = gx * mh + jm, tn = gy * nh + (j - jm * nh);
  if (jm >= mh || tm >= ntm || tn >= ntn) return;
  const int m0 = tm * BM, n0 = tn * BN;
  const int nst = p.Kq / kBK;

  // (rows past M read as zeros from past the buffer; weight rows are padded to 256)
  const i32x4 xr = buffer_rsrc(p.x + (int64_t)m0 * p.Kq, min(BM, p.M - m0) * p.Kq);
  const i32x4 wr = buffer_rsrc(p.w + (int64_t)n0 * p.Kq, BN * p.Kq);
  uint32_t avoff[AR], wvoff[BR];
#pragma unroll
  for (int i = 0; i < AR; ++i) avoff[i] = (uint32_t)((r0 + i * kRowsPerPass) * p.Kq + cva * 16);
#pragma unroll
  for (int i = 0; i < BR; ++i) wvoff[i] = (uint32_t)((r0 + i * kRowsPerPass) * p.Kq + cvb * 16);
  int issued = 0;
  auto fill = [&](int slot, auto q_tag) {
    constexpr int q = decltype(q_tag)::value;
    uint4* dst = ring + slot * STAGE;
    const bool live = issued < nst;
    if constexpr (q < AR)
      lds_fill16(xr, __builtin_amdgcn_readfirstlane(lds_addr(dst + (q * kRowsPerPass + wave * 8) * kCH)),
                 live ? avoff[q] + (uint32_t)(issued * kBK) : kOOB);
    else
      lds_fill16(wr, __builtin_amdgcn_readfirstlane(lds_addr(dst + (BM + (q - AR) * kRowsPerPass + wave * 8) * kCH)),
                 live ? wvoff[q - AR] + (uint32_t)(issued * kBK) : kOOB);
  };

  i32x4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int k = 0; k < TM; ++k) acc[i][k] = i32x4{0, 0, 0, 0};

  const int lr = lane & 15, lc = lane >> 4;
  int arow[2], brow[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    arow[ks] = (wm * WTM + lr) * kCH + ((ks * 4 + lc) ^ (lr & 7));
    // MFMA row r of channel tile i is channel 32 (i / 2) + 8 (r / 4) + 4 (i % 2) + r % 4, so that a
    // pair of tiles leaves 8 consecutive channels of a row in a lane
    brow[ks] = (BM + wn * WTN + 8 * (lr >> 2) + (lr & 3)) * kCH + ((ks * 4 + lc) ^ ((lr & 3) | (lr & 4)));
  }
  struct Frags {
    uint4 a[TN], b[TM];
  };
  constexpr int NR = TN + TM;
  auto read1 = [&](Frags& f, int slot, auto ks_tag, auto q_tag) {
    constexpr int ks = decltype(ks_tag)::value, q = decltype(q_tag)::value;
    const uint4* st = ring + slot * STAGE;
    if constexpr (q < TN)
      f.a[q] = st[brow[ks] + ((q >> 1) * 32 + (q & 1) * 4) * kCH];
    else
      f.b[q - TN] = st[arow[ks] + (q - TN) * 16 * kCH];
  };
  auto phase = [&](const Frags& cur, Frags& nxt, int rslot, auto ks_tag, int fslot, auto fill_tag) {
    constexpr bool FILL = decltype(fill_tag)::value;
    constexpr int RG = TM > 4 ? TM - 2 : TM;
    static_for<0, TM>([&](auto jj) {
      constexpr int k = decltype(jj)::value;
#pragma unroll
      for (int i = 0; i < TN; ++i) acc[i][k] = mma(cur.a[i], cur.b[k], acc[i][k]);
      static_for<0, NR>([&](auto q) {
        if constexpr (decltype(q)::value * RG / NR == k) read1(nxt, rslot, ks_tag, q);
      });
      if constexpr (FILL)
        static_for<0, LPS>([&](auto q) {
          if constexpr (decltype(q)::value * TM / LPS == k) fill(fslot, q);
        });
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  static_for<0, NS>([&](auto i) {
    static_for<0, LPS>([&](auto q) { fill(decltype(i)::value, q); });
    ++issued;
  });
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((NS - 1) * LPS) : "memory");
  Frags f0, f1;
  constexpr std::integral_constant<int, 0> k0{};
  constexpr std::integral_constant<int, 1> k1{};
  static_for<0, NR>([&](auto q) { read1(f0, 0, k0, q); });
  int slot = 0;
  for (int t = 0; t < nst; ++t) {
    const int next = slot + 1 == NS ? 0 : slot + 1;
    phase(f0, f1, slot, k1, 0, std::false_type{});
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NS - 2) * LPS) : "memory");
    phase(f1, f0, next, k0, slot, std::true_type{});
    ++issued;
    slot = next;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  const ActClamp ac = act_clamp_of(p.act, p.alpha);
  auto epilogue = [&](auto mode_tag) {
#pragma unroll
    for (int pr = 0; pr < TN / 2; ++pr) {
      const int n = n0 + wn * WTN + pr * 32 + lc * 8;
      if (n >= p.N) continue;
      float ws[8], bias[8];
      load8f(p.ws + n, ws);
      if (p.bias) {
        load8f(p.bias + n, bias);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[e] = 0.0f;
      }
#pragma unroll
      for (int k = 0; k < TM; ++k) {
        const int m = m0 + wm * WTM + k * 16 + lr;
        if (m >= p.M) continue;
        int a[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = acc[2 * pr + (e >> 2)][k][e & 3];
        finish8<F32, decltype(mode_tag)::value>(p, a, p.xs[m], ws, bias, m, n, ac);
      }
    }
  };
  if (act_mode(p.act) == 1)
    epilogue(std::integral_constant<int, 1>{});
  else if (act_mode(p.act) == 0)
    epilogue(std::integral_constant<int, 0>{});
  else
    epilogue(std::integral_constant<int, 2>{});
}

template <int BM, int BN, int WM, int WN, int NS, bool F32>
hipError_t launch_one(QDenseParams p, hipStream_t s) {
  // the split of the tile grid over the XCDs that has each fetch the fewest operand rows
  const int ntm = (p.M + BM - 1) / BM, ntn = (p.N + BN - 1) / BN;
  int64_t best = INT64_MAX, blocks = 0;
  for (int py = 1; py <= 8; py *= 2) {
    const int mh = (ntm + 8 / py - 1) / (8 / py), nh = (ntn + py - 1) / py;
    const int64_t cost = (int64_t)mh * nh * 4096 + mh * BM + nh * BN;  // (first of all no XCD with more tiles)
    if (cost < best) best = cost, p.py = py, blocks = 8 * (int64_t)mh * nh;
  }
  qdense_kernel<BM, BN, WM, WN, NS, F32><<<(unsigned)blocks, 64 * WM * WN, 0, s>>>(p);
  return hipGetLastError();
}

#define BYOC_QDENSE_TILES(X) \
  X(256, 256, 2, 4, 2)       \
  X(128, 128, 2, 2, 3)       \
  X(64, 64, 2, 2, 4)

}  // namespace

hipError_t launch_quant_rows(const QRowsParams& p, hipStream_t s) {
  if (p.rows < 1 || p.Kq % 128 != 0 || p.K > p.Kq) return hipErrorInvalidValue;
  if (p.f32) quant_rows<true>(p, s);
  else quant_rows<false>(p, s);
  return hipGetLastError();
}

// The largest tile that leaves every CU one.
QDenseTile choose_qdense_tile(int64_t M, int64_t N) {
  for (int b : {256, 128})
    if (((M + b - 1) / b) * ((N + b - 1) / b) >= 256) return {b, b};
  return {64, 64};
}

hipError_t launch_qdense(const QDenseParams& p, QDenseTile t, hipStream_t s) {
#define X(BM, BN, WM, WN, NS)           \
  if (t.bm == BM && t.bn == BN)         \
    return p.f32 ? launch_one<BM, BN, WM, WN, NS, true>(p, s) : launch_one<BM, BN, WM, WN, NS, false>(p, s);
  BYOC_QDENSE_TILES(X)
#undef X
  return hipErrorInvalidValue;
}

}  // namespace byoc
