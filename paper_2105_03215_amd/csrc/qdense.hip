// Dense composite on 8-bit codes with a scale for each token and each output
// channel: the rows of the activations are quantized on the way in (quant_rows),
// multiplied on int8 MFMA with exact int32 sums, and rescaled in the epilogue.
//
//   a_m = max_k |x_mk|,  q_mk = rint(127 x_mk / a_m),
//   y_mn = act((sum_k q_mk r_nk) (a_m / 127) (b_n / 127) + bias_n + res_mn)
//
// with r, b the same of the weight rows, formed once at engine creation by the
// same kernel.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "lds_dma.h"
#include "dense_epilogue.h"

namespace byoc {
namespace {

using namespace dma;

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

// WPR waves per row; NC > 0: the row's chunks of 8 stay in registers as they came
// between the maximum and the codes (at most NC per lane), NC = 0: they are read
// twice.  HBM bound: 8192 rows of 4096 bf16, 101 MB, in 19.9 us (5.1 TB/s;
// 21.8 with a wave per row).
template <bool F32, int WPR, int NC>
__global__ __launch_bounds__(256) void quant_rows_kernel(QRowsParams p) {
  constexpr int LANES = 64 * WPR;
  __shared__ uint32_t tops[4];
  const int tid = threadIdx.x, wave = tid >> 6;
  const int row = blockIdx.x * (4 / WPR) + tid / LANES;
  const int lane = tid % LANES;
  const int chunks = p.Kq / 8;
  const int K = row < p.M ? p.K : 0;
  const int64_t at = (int64_t)row * p.ldx;
  uint32_t top = 0;
  Chunk<F32> v[NC > 0 ? NC : 1];
  auto widen = [&](const Chunk<F32>& c) {
    float f[8];
    c.get(f);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7FFFFFFFu);
  };
  if constexpr (NC > 0) {
#pragma unroll
    for (int i = 0; i < NC; ++i) v[i].load(p.x, at, (i * LANES + lane) * 8, K);
#pragma unroll
    for (int i = 0; i < NC; ++i) widen(v[i]);
  } else {
    for (int c = lane; c < chunks; c += LANES) {
      v[0].load(p.x, at, c * 8, K);
      widen(v[0]);
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
  if constexpr (WPR > 1) {
    if ((tid & 63) == 0) tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WPR; ++w) top = max(top, tops[wave / WPR * WPR + w]);
  }
  if (row >= p.rows) return;
  const RowScale r = row_scale(top);
  if (lane == 0) p.scale[row] = r.scale;
  int8_t* q = p.q + (int64_t)row * p.Kq;
  auto write = [&](int c, const Chunk<F32>& x) {
    float f[8], y[8];
    x.get(f);
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
      v[0].load(p.x, at, c * 8, K);
      write(c, v[0]);
    }
  }
}

template <bool F32, int WPR, int NC>
void quant_rows_as(const QRowsParams& p, hipStream_t s) {
  quant_rows_kernel<F32, WPR, NC><<<(p.rows + 4 / WPR - 1) / (4 / WPR), 256, 0, s>>>(p);
}
template <bool F32>
void quant_rows(const QRowsParams& p, hipStream_t s) {
  const int c = p.Kq / 8;  // chunks of a row
  if (c <= 64) quant_rows_as<F32, 1, 1>(p, s);
  else if (c <= 128) quant_rows_as<F32, 1, 2>(p, s);
  else if (c <= 512) quant_rows_as<F32, 4, 2>(p, s);
  else if (c <= 1024) quant_rows_as<F32, 4, 4>(p, s);
  else quant_rows_as<F32, 4, 0>(p, s);
}

constexpr int kCH = 8;   // 16-byte chunks of an LDS row
constexpr int kBK = 128;  // codes of a stage

__device__ __forceinline__ i32x4 mma(uint4 a, uint4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// Eight columns of one output row: y = act(acc * scale + bias + res).  The sum meets the
// channel's scale first: the product of the two scales alone may leave float32 where the result
// does not (rows of 2^-64 under weights of 2^-64: the product of the scales has 7 bits left).
template <bool F32, int MODE>
__device__ __forceinline__ void finish8(const QDenseParams& p, const int* acc, float xs, const float* ws,
                                        const float* bias, const Chunk<F32>& res, int64_t m, int n, ActClamp ac) {
  float r[8], v[8];
  res.get(r);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = act_nan<F32, MODE>(__builtin_fmaf((float)acc[e] * ws[e], xs, bias[e]) + r[e], ac);
  store_chunk<F32>(p.y, m * p.ldy, n, p.N, v);  // (a row of the caller's, of any width, ends where it ends)
}

// BM rows x BN channels per workgroup of WM x WN waves; both operands streamed
// HBM -> LDS in stages of 128 codes through a ring of NS, the MFMA operands of a
// step of 64 codes read while the previous step multiplies.  Bound by the wait at the end of a stage (below,
// at the tiles): 8192 x 4096 x 8192 256 us, 2.1 POP/s.
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

  // XCD x = (gx, gy) of 8 / py x py owns a block of the tile grid (workgroup b runs on XCD b % 8) and
  // walks it in bands of 4 row tiles: the 32 tiles that its CUs have at a time then share 4 row and 8
  // channel tiles in its L2 (8192 x 4096 x 8192: 260 us row by row, 256 in bands of 4, 277 of 8)
  constexpr int kBand = 4;
  const int ntm = (p.M + BM - 1) / BM, ntn = (p.N + BN - 1) / BN;
  const int x = blockIdx.x & 7, j = blockIdx.x >> 3;
  const int px = 8 / p.py;
  const int mh = (ntm + px - 1) / px, nh = (ntn + p.py - 1) / p.py;
  const int gx = x / p.py, gy = x - gx * p.py;
  const int band = j / (kBand * nh), at = j - band * kBand * nh;
  const int bm = min(kBand, mh - band * kBand);
  if (bm <= 0) return;
  const int jn = at / bm;
  const int tm = gx * mh + band * kBand + at - jn * bm, tn = gy * nh + jn;
  if (jn >= nh || tm >= ntm || tn >= ntn) return;
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

  // Epilogue: lane = row lr of each row tile, 8 consecutive channels per pair of channel tiles; the
  // residuals of a batch of rows are on their way together
  const ActClamp ac = act_clamp_of(p.act, p.alpha);
  // (bf16: 8192 x 4096 x 8192 314 us one by one, 290 together; fp32, twice the registers: 1531 x 1000 x 2056
  // 19.9 and 21.0)
  constexpr int BATCH = F32 ? 1 : TM;
  float xs[TM];
#pragma unroll
  for (int k = 0; k < TM; ++k) {
    const int m = m0 + wm * WTM + k * 16 + lr;
    xs[k] = m < p.M ? p.xs[m] : 0.0f;
  }
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
      for (int k0 = 0; k0 < TM; k0 += BATCH) {
        Chunk<F32> res[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
          res[k] = load_res<F32>(p, min(m0 + wm * WTM + (k0 + k) * 16 + lr, p.M - 1), n);
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
          const int m = m0 + wm * WTM + (k0 + k) * 16 + lr;
          if (m >= p.M) continue;
          int a[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] = acc[2 * pr + (e >> 2)][k0 + k][e & 3];
          finish8<F32, decltype(mode_tag)::value>(p, a, xs[k0 + k], ws, bias, res[k], m, n, ac);
        }
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

// Few rows: a workgroup of 8 waves owns 16 NT channels and all rows and splits the
// reduction over its waves, operands straight to registers, the waves' sums joined
// in LDS; the time is that of reading the weights.  MT tiles of 16 rows.
//
// FUSED: the rows are quantized by every workgroup for itself, into LDS, while its
// first weights are on their way; that saves the launch that would do it.
constexpr int kRowWaves = 8;
constexpr int kRowThreads = 64 * kRowWaves;
constexpr int kRowSteps = 4;                // steps of 64 codes per wave with loads in flight together
constexpr int kFusedCodes = 16 * kRowThreads;  // codes of all rows that FUSED takes

template <int MT, int NT, bool F32, bool FUSED>
__global__ __launch_bounds__(kRowThreads) void qdense_rows_kernel(QDenseParams p, QRowsParams q) {
  __shared__ i32x4 red[kRowWaves][MT * NT][64];
  __shared__ __align__(16) int8_t codes[FUSED ? kFusedCodes : 16];
  __shared__ float scales[16];
  __shared__ uint32_t tops[kRowWaves];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lc = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16 * NT;
  const int steps = p.Kq / 64;
  // a wave takes pairs of steps, 128 bytes of each weight row: wave w steps 2w, 2w + 1, 2w + 16, ...
  auto step_of = [&](int i) { return (i >> 1) * 2 * kRowWaves + 2 * wave + (i & 1); };
  const int8_t* wp = p.w + (int64_t)(n0 + lr) * p.Kq + lc * 16;
  uint4 a[kRowSteps][NT];
  auto load_w = [&](int i0) {
#pragma unroll
    for (int u = 0; u < kRowSteps; ++u) {
      const int t = step_of(i0 + u);
#pragma unroll
      for (int j = 0; j < NT; ++j)
        a[u][j] = t < steps ? *(const uint4*)(wp + (int64_t)j * 16 * p.Kq + t * 64) : make_uint4(0u, 0u, 0u, 0u);
    }
  };
  // this thread's 8 outputs, and what they need besides the sums: on its way from the start
  static_assert(MT * 16 * NT * 2 <= kRowThreads, "an output group each");
  const int om = tid / (NT * 2), og = tid % (NT * 2), on = n0 + og * 8;
  const bool out = om < p.M && on < p.N && tid < MT * 16 * NT * 2;
  float ws[8], bias[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  Chunk<F32> res;
  load_w(0);
  if (out) {
    load8f(p.ws + on, ws);
    if (p.bias) load8f(p.bias + on, bias);
    res = load_res<F32>(p, om, on);
  }
  if constexpr (FUSED) {
    // waves per row: as many as there are for the rows rounded up to a power of two
    const int lg = p.M > 4 ? 3 : (p.M > 2 ? 2 : p.M - 1);
    const int wpr = kRowWaves >> lg;
    const int row = wave / wpr, part = (wave % wpr) * 64 + lane;
    const bool live = row < p.M;
    const int chunks = p.Kq / 8;
    constexpr int NC = 4;  // (2 kFusedCodes / kRowThreads / 8)
    Chunk<F32> v[NC];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      v[i].load(q.x, (int64_t)row * q.ldx, (i * wpr * 64 + part) * 8, live ? q.K : 0);
      float f[8];
      v[i].get(f);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7FFFFFFFu);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    for (int w = 0; w < wpr; ++w) top = max(top, tops[row * wpr + w]);
    const RowScale r = row_scale(top);
    if (live && part == 0) scales[row] = r.scale;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int c = i * wpr * 64 + part;
      if (!live || c >= chunks) continue;
      float f[8], y[8];
      v[i].get(f);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = code_of<F32>(f[e], r);
      *(uint2*)(codes + row * p.Kq + c * 8) = make_uint2(pack_codes(y), pack_codes(y + 4));
    }
    __syncthreads();
  }
  i32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  for (int i0 = 0; step_of(i0) < steps; i0 += kRowSteps) {
    uint4 b[kRowSteps][MT];
#pragma unroll
    for (int u = 0; u < kRowSteps; ++u) {
      const int t = step_of(i0 + u);
#pragma unroll
      for (int k = 0; k < MT; ++k) {
        const int m = k * 16 + lr;
        const int8_t* xp = (FUSED ? codes : p.x) + (int64_t)m * p.Kq + t * 64 + lc * 16;
        b[u][k] = m < p.M && t < steps ? *(const uint4*)xp : make_uint4(0u, 0u, 0u, 0u);
      }
    }
    uint4 w[kRowSteps][NT];
#pragma unroll
    for (int u = 0; u < kRowSteps; ++u)
#pragma unroll
      for (int j = 0; j < NT; ++j) w[u][j] = a[u][j];
    load_w(i0 + kRowSteps);
#pragma unroll
    for (int u = 0; u < kRowSteps; ++u)
#pragma unroll
      for (int k = 0; k < MT; ++k)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[k][j] = mma(w[u][j], b[u][k], acc[k][j]);
  }
#pragma unroll
  for (int k = 0; k < MT; ++k)
#pragma unroll
    for (int j = 0; j < NT; ++j) red[wave][k * NT + j][lane] = acc[k][j];
  __syncthreads();
  // row m, channels n0 + 16 j + 4 c .. + 3 sit in lane 16 c + m % 16 of tile (m / 16, j) of every wave
  if (!out) return;
  const ActClamp ac = act_clamp_of(p.act, p.alpha);
  int sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const i32x4 r = red[w][(om >> 4) * NT + (og >> 1)][((og & 1) * 2 + half) * 16 + (om & 15)];
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[4 * half + e] += r[e];
    }
  const float xs = FUSED ? scales[om] : p.xs[om];
  auto epilogue = [&](auto mode_tag) {
    finish8<F32, decltype(mode_tag)::value>(p, sum, xs, ws, bias, res, om, on, ac);
  };
  if (act_mode(p.act) == 1)
    epilogue(std::integral_constant<int, 1>{});
  else if (act_mode(p.act) == 0)
    epilogue(std::integral_constant<int, 0>{});
  else
    epilogue(std::integral_constant<int, 2>{});
}

template <bool F32>
hipError_t launch_rows(const QDenseParams& p, const QRowsParams& q, bool fused, hipStream_t s) {
  const int mt = (p.M + 15) / 16;
  const int nt = 1;
  const dim3 grid((p.N + 16 * nt - 1) / (16 * nt));
  if (fused) qdense_rows_kernel<1, 1, F32, true><<<grid, kRowThreads, 0, s>>>(p, q);
  else if (mt == 1) qdense_rows_kernel<1, 1, F32, false><<<grid, kRowThreads, 0, s>>>(p, q);
  else if (mt == 2) qdense_rows_kernel<2, 1, F32, false><<<grid, kRowThreads, 0, s>>>(p, q);
  else return hipErrorInvalidValue;
  return hipGetLastError();
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

// Tiles (BM, BN, waves along each, ring stages) and what they cost in microseconds:
// a stage of 128 codes while at most one workgroup runs per CU or all slots (occ per
// CU) are busy, and a round's prologue and epilogue.  Fitted to 15 shapes from 24 x 4096 x
// 12288 to 8192 x 4096 x 8192, on which the choice is never more than 8% behind the
// fastest tile (18 others: 18% at 700 x 128 x 700, 16% at 284 x 5549 x 10785, else up to 10%).  A 256x256 stage, 64 KB from
// L2 to LDS and 192 KB from LDS to registers, takes 1.8 us for 0.9 us of matrix operations: in
// 8192 x 4096 x 8192 the matrix cores are busy for 56% of the cycles, the LDS for 21%, and a third of the
// waves' time is waiting at the end of a stage, for its loads and its barrier, with a ring of two.  With 4 waves of 128 x
// 128 the LDS reads fall by a third, but one wave per SIMD hides nothing (347 us against 256), and
// half-depth stages in a ring of five fetch half cache lines (285).
//   id BM BN WM WN NS  occ  lone  busy  round
#define BYOC_QDENSE_TILES(X)                 \
  X(0, 256, 256, 2, 4, 2, 1, 1.33, 1.8, 9.0) \
  X(1, 256, 128, 4, 2, 3, 1, 0.77, 1.0, 6.0) \
  X(2, 128, 128, 2, 4, 3, 1, 0.51, 0.6, 4.2) \
  X(3, 128, 128, 2, 4, 2, 2, 0.71, 1.09, 5.0) \
  X(4, 128, 64, 4, 2, 3, 2, 0.39, 0.70, 3.5) \
  X(5, 64, 64, 2, 2, 4, 2, 0.33, 0.46, 2.3)  \
  X(6, 32, 32, 2, 1, 8, 2, 0.26, 0.30, 1.8)

double tile_cost(int bm, int bn, int occ, double lone, double busy, double round, int64_t M, int64_t N, int64_t Kq) {
  const int64_t tiles = ((M + bm - 1) / bm) * ((N + bn - 1) / bn), slots = 256 * occ;
  const double stages = (double)(Kq / kBK);
  const int64_t rest = tiles % slots;
  double t = (double)(tiles / slots) * (stages * busy + round);
  if (rest) t += stages * (rest <= (occ == 1 ? 128 : 256) ? lone : busy) + round;
  return t;
}

}  // namespace

hipError_t launch_quant_rows(const QRowsParams& p, hipStream_t s) {
  if (p.rows < 1 || p.Kq % 128 != 0 || p.K > p.Kq) return hipErrorInvalidValue;
  if (p.f32) quant_rows<true>(p, s);
  else quant_rows<false>(p, s);
  return hipGetLastError();
}

constexpr int kRowsN = 16 * 256;  // channels of the rows kernel: a workgroup of 16 for each CU

// (1 x 4096 x 4096: 8.4 us, 8.7 with a launch for the rows; 8 x 1024 x 4096: 5.3 and 7.9; but 4 x 4096 x 4096,
// as every workgroup quantizes all rows, 12.5 and 8.9, and 1 x 4096 x 12288, 768 workgroups, 18.5 and 12.5 on
// 64x64 tiles)
bool qdense_fuses_rows(int64_t M, int64_t N, int64_t Kq) { return M <= 8 && M * Kq <= kFusedCodes && N <= kRowsN; }

hipError_t launch_qdense_fused(const QDenseParams& p, const QRowsParams& q, hipStream_t s) {
  if (!qdense_fuses_rows(p.M, p.N, p.Kq)) return hipErrorInvalidValue;
  return p.f32 ? launch_rows<true>(p, q, true, s) : launch_rows<false>(p, q, true, s);
}

// The rows kernel where all of its workgroups run at once, one per CU (32 x 768 x
// 3072: 8.8 us against 9.4 on 32x32 tiles, 16 x 8192 x 1024: 15.0 against 16.4; but 16 x
// 4096 x 12288, 768 workgroups: 23.5 against 15.2); else the tile of least modelled time.
QDenseTile choose_qdense_tile(int64_t M, int64_t N, int64_t Kq) {
  if (M <= 32 && N <= kRowsN) return {kQDenseRows, (int)(M + 15) / 16 * 16, 16, 0};
  QDenseTile best{};
  double least = INFINITY;
#define X(ID, BM, BN, WM, WN, NS, OCC, LONE, BUSY, ROUND)                                                \
  if (const double c = tile_cost(BM, BN, OCC, LONE, BUSY, ROUND, M, N, Kq); c < least) least = c, best = {ID, BM, BN, NS};
  BYOC_QDENSE_TILES(X)
#undef X
  return best;
}

bool qdense_tile_of(int id, QDenseTile* t) {
#define X(ID, BM, BN, WM, WN, NS, OCC, LONE, BUSY, ROUND) \
  if (id == ID) return *t = {ID, BM, BN, NS}, true;
  BYOC_QDENSE_TILES(X)
#undef X
  return false;
}

hipError_t launch_qdense(const QDenseParams& p, QDenseTile t, hipStream_t s) {
  if (t.id == kQDenseRows) return p.f32 ? launch_rows<true>(p, {}, false, s) : launch_rows<false>(p, {}, false, s);
#define X(ID, BM, BN, WM, WN, NS, OCC, LONE, BUSY, ROUND) \
  if (t.id == ID) return p.f32 ? launch_one<BM, BN, WM, WN, NS, true>(p, s) : launch_one<BM, BN, WM, WN, NS, false>(p, s);
  BYOC_QDENSE_TILES(X)
#undef X
  return hipErrorInvalidValue;
}

}  // namespace byoc
