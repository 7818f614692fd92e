// Dense composite on microscaled 4-bit floating point: blocks of 32 values along the
// reduction share a power of two, the values over it are rounded to 4 bits.  The rows of the
// activations are quantized on the way in (mx_rows), multiplied on the scaled matrix
// instructions, which take a block's power of two with its codes, and summed in float32:
//
//   y_mn = act(sum_c 2^(s_mc + t_nc) sum_{k in block c} q_mk r_nk + bias_n + res_mn)
//
// with r, t the same of the weight rows, formed once at engine creation by the same kernel.
// A block's scale is a power of two and every product of two codes a multiple of 1/4 of at
// most 36, so that only the float32 sum rounds.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "dense_epilogue.h"
#include "lds_dma.h"

namespace byoc {
namespace {

using namespace dma;

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// Where the scale of row r's block c stands.  A stage of 256 codes of 32 rows has 64 words of
// scales, one for each lane of a wave: lane 16 (c % 4) + 4 (r % 32 / 8) + r % 4 has those of rows
// r and r + 4, each for the stage's two steps of 128 codes.
__device__ __forceinline__ int64_t mx_scale_at(int64_t r, int c, int Kq) {
  const int lr = (int)(r % 32) / 8 * 4 + (int)(r % 4);
  return ((r / 32 * (Kq / 256) + c / 8) * 64 + c % 4 * 16 + lr) * 4 + (r / 4 % 2) * 2 + c / 4 % 2;
}

// The magnitudes' largest bits of 8 values.  They are compared as integers, which orders NaN
// above infinity above every number.
template <bool F32>
__device__ __forceinline__ uint32_t top_bits(const Chunk<F32>& c) {
  uint32_t top = 0;
  if constexpr (F32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(c.v[e]) & 0x7FFFFFFFu);
  } else {
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    u16x2 m = {0, 0};
    for (uint32_t w : {c.u.x, c.u.y, c.u.z, c.u.w})
      m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu));
    top = (uint32_t)max(m[0], m[1]) << 16;
  }
  return top;
}
// A block's scale byte from the bits of its largest magnitude, and the power of two that it says (2^-127 has
// no normal form; the byte of an infinite or NaN block is never used as a power).
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
  const uint32_t e = bits >> 23;
  return e == 255u ? 255u : max(e, 2u) - 2u;
}
__device__ __forceinline__ float scale_power(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }
// 8 codes of a block.
template <bool F32>
__device__ __forceinline__ uint32_t codes_of(const Chunk<F32>& c, float power) {
  uint32_t w = 0;
  if constexpr (F32) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c.v[0], c.v[1], power, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c.v[2], c.v[3], power, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c.v[4], c.v[5], power, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c.v[6], c.v[7], power, 3);
  } else {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, c.u.x), power, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, c.u.y), power, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, c.u.z), power, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, c.u.w), power, 3);
  }
  return w;
}
// The largest over the 4 lanes that share a block.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));  // lanes 1 0 3 2
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));  // 2 3 0 1
}

// 32 rows x a stage of 256 codes per workgroup, 4 lanes of 8 values to a block; the stage's
// scales leave as whole words through LDS.
template <bool F32>
__global__ __launch_bounds__(256) void mx_rows_kernel(MxRowsParams p) {
  __shared__ uint32_t words[64];
  const int tid = threadIdx.x, nst = p.Kq / 256;
  const int rg = blockIdx.x / nst, st = blockIdx.x - rg * nst;
  const int c = tid & 31, col = st * 256 + c * 8;
  Chunk<F32> v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = rg * 32 + i * 8 + (tid >> 5);
    v[i].load(p.x, (int64_t)row * p.ldx, col, row < p.M ? p.K : 0);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i * 8 + (tid >> 5);
    const uint32_t byte = scale_byte(quad_max(top_bits(v[i])));
    *(uint32_t*)(p.q + (int64_t)(rg * 32 + r) * (p.Kq / 2) + col / 2) = codes_of(v[i], scale_power(byte));
    if ((c & 3) == 0) ((uint8_t*)words)[mx_scale_at(r, c >> 2, 256)] = (uint8_t)byte;
  }
  __syncthreads();
  if (tid < 64) ((uint32_t*)p.scale)[(int64_t)blockIdx.x * 64 + tid] = words[tid];
}

constexpr int kCH = 8;         // 16-byte chunks of an LDS row
constexpr int kStageK = 256;   // codes of a stage: 128 bytes of a row

// D += A B of 128 codes, each with the scale byte SA / SB of its lane's word.
template <int SA, int SB>
__device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c, uint32_t sa, uint32_t sb) {
  const i32x8 a8 = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  const i32x8 b8 = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, SA, (int)sa, SB, (int)sb);
}

// 4 bytes per lane from a buffer straight into LDS (the form of lds_fill16).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_fill4(i32x4 rsrc, uint32_t lds_addr, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds"
               :
               : "s"(lds_addr), "v"(voff), "s"(rsrc)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// Eight columns of one output row.
template <bool F32, int MODE, class P>
__device__ __forceinline__ void finish8(const P& p, const float* acc, const float* bias, const Chunk<F32>& res, int64_t m,
                                        int n, ActClamp ac) {
  float r[8], v[8];
  res.get(r);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = act_nan<F32, MODE>(acc[e] + bias[e] + r[e], ac);
  store_chunk<F32>(p.y, m * p.ldy, n, p.N, v);
}

// BM rows x BN channels per workgroup of WM x WN waves; codes and scales of both operands streamed
// HBM -> LDS in stages of 256 codes through a ring of NS, the MFMA operands of a step of 128 codes read
// while the previous step multiplies.  Both operands' rows are permuted within 32 (MFMA row r of tile i is
// row 32 (i / 2) + 8 (r / 4) + 4 (i % 2) + r % 4): a lane then has one word of scales for a pair of tiles
// and a stage, and 8 consecutive channels of an output row.
template <int BM, int BN, int WM, int WN, int NS, bool F32>
__global__ __launch_bounds__(64 * WM * WN) void mxdense_kernel(MxDenseParams p) {
  constexpr int kNT = 64 * WM * WN, NW = WM * WN;
  constexpr int kRowsPerPass = kNT / kCH;
  constexpr int WTM = BM / WM, WTN = BN / WN;
  constexpr int TM = WTM / 16, TN = WTN / 16;
  constexpr int AR = BM / kRowsPerPass, BR = BN / kRowsPerPass;
  constexpr int GM = BM / 32, GN = BN / 32;      // groups of 32 rows: 256 bytes of scales a stage each
  constexpr int SR = (GM + GN + NW - 1) / NW;    // of them a wave
  static_assert(BM % kRowsPerPass == 0 && BN % kRowsPerPass == 0 && kRowsPerPass % 16 == 0, "fill shape");
  static_assert(WTM % 16 == 0 && WTN % 32 == 0, "wave tile: whole MFMA rows, pairs of channel tiles");
  static_assert(TM % 2 == 0 || (TM == 1 && WM == 2), "row tiles in pairs");
  constexpr int LPS = AR + BR + SR;
  constexpr int CODES = (BM + BN) * kCH;           // uint4 per stage
  constexpr int STAGE = CODES + SR * NW * 16;      // with the scales
  static_assert(NS >= 2 && (NS - 1) * LPS <= 63, "vmcnt immediate");
  static_assert(NS * STAGE * 16 <= kLdsLimit, "LDS");
  __shared__ uint4 ring[NS * STAGE];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int r0 = tid / kCH;
  const int cv = (lane & 7) ^ ((r0 & 3) | ((r0 & 8) >> 1));

  // XCD x = (gx, gy) of 8 / py x py owns a block of the tile grid (workgroup b runs on XCD b % 8) and
  // walks it in bands of 4 row tiles
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
  const int nst = p.Kq / kStageK, rb = p.Kq / 2;  // bytes of a row of codes

  // (rows past M and their scales read as zeros from past the buffer; weight rows are padded to 256)
  const int live_groups = (min(BM, p.M - m0) + 31) / 32;
  const i32x4 xr = buffer_rsrc(p.x + (int64_t)m0 * rb, min(BM, p.M - m0) * rb);
  const i32x4 wr = buffer_rsrc(p.w + (int64_t)n0 * rb, BN * rb);
  const i32x4 xsr = buffer_rsrc(p.xs + (int64_t)(m0 / 32) * nst * 256, live_groups * nst * 256);
  const i32x4 wsr = buffer_rsrc(p.ws + (int64_t)(n0 / 32) * nst * 256, GN * nst * 256);
  uint32_t avoff[AR], wvoff[BR], svoff[SR];
#pragma unroll
  for (int i = 0; i < AR; ++i) avoff[i] = (uint32_t)((r0 + i * kRowsPerPass) * rb + cv * 16);
#pragma unroll
  for (int i = 0; i < BR; ++i) wvoff[i] = (uint32_t)((r0 + i * kRowsPerPass) * rb + cv * 16);
#pragma unroll
  for (int i = 0; i < SR; ++i) {  // (uniform over a wave but for the lane)
    const int g = i * NW + wave;
    svoff[i] = g < GM + GN ? (uint32_t)((g < GM ? g : g - GM) * nst * 256 + lane * 4) : kOOB;
  }
  int issued = 0;
  auto fill = [&](int slot, auto q_tag) {
    constexpr int q = decltype(q_tag)::value;
    uint4* dst = ring + slot * STAGE;
    const bool live = issued < nst;
    if constexpr (q < AR) {
      lds_fill16(xr, __builtin_amdgcn_readfirstlane(lds_addr(dst + (q * kRowsPerPass + wave * 8) * kCH)),
                 live ? avoff[q] + (uint32_t)(issued * 128) : kOOB);
    } else if constexpr (q < AR + BR) {
      lds_fill16(wr, __builtin_amdgcn_readfirstlane(lds_addr(dst + (BM + (q - AR) * kRowsPerPass + wave * 8) * kCH)),
                 live ? wvoff[q - AR] + (uint32_t)(issued * 128) : kOOB);
    } else {
      constexpr int i = q - AR - BR;
      const int g = i * NW + wave;
      lds_fill4(g < GM ? xsr : wsr, __builtin_amdgcn_readfirstlane(lds_addr(dst + CODES + g * 16)),
                live ? svoff[i] + (uint32_t)(issued * 256) : kOOB);
    }
  };

  f32x4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int k = 0; k < TM; ++k) acc[i][k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const int lr = lane & 15, lc = lane >> 4;
  const int prow = 8 * (lr >> 2) + (lr & 3);
  constexpr bool LONE = TM == 1;  // (a wave has one tile of a pair of row tiles)
  const int wrow = LONE ? 4 * wm : wm * WTM;
  int arow[2], brow[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    const int ch = (ks * 4 + lc) ^ ((lr & 3) | (lr & 4));
    arow[ks] = (wrow + prow) * kCH + ch;
    brow[ks] = (BM + wn * WTN + prow) * kCH + ch;
  }
  struct Frags {
    uint4 a[TN], b[TM];
  };
  constexpr int PM = (TM + 1) / 2, PN = TN / 2;
  struct Scales {
    uint32_t a[PN], b[PM];
  };
  constexpr int NR = TN + TM;
  auto read1 = [&](Frags& f, int slot, auto ks_tag, auto q_tag) {
    constexpr int ks = decltype(ks_tag)::value, q = decltype(q_tag)::value;
    const uint4* st = ring + slot * STAGE;
    if constexpr (q < TN)
      f.a[q] = st[brow[ks] + ((q >> 1) * 32 + (q & 1) * 4) * kCH];
    else
      f.b[q - TN] = st[arow[ks] + (((q - TN) >> 1) * 32 + ((q - TN) & 1) * 4) * kCH];
  };
  auto read_scales = [&](Scales& s, int slot) {
    const uint32_t* at = (const uint32_t*)(ring + slot * STAGE + CODES) + lane;
#pragma unroll
    for (int i = 0; i < PN; ++i) s.a[i] = at[(GM + wn * (WTN / 32) + i) * 64];
#pragma unroll
    for (int i = 0; i < PM; ++i) s.b[i] = at[((LONE ? 0 : wm * (WTM / 32)) + i) * 64];
    if constexpr (LONE) s.b[0] >>= 16 * wm;
  };
  auto phase = [&](const Frags& cur, const Scales& sc, Frags& nxt, int rslot, auto ks_tag, int fslot, auto fill_tag) {
    constexpr bool FILL = decltype(fill_tag)::value;
    constexpr int ks = 1 - decltype(ks_tag)::value;  // of the step that multiplies
    constexpr int RG = TM > 4 ? TM - 2 : TM;
    static_for<0, TM>([&](auto jj) {
      constexpr int k = decltype(jj)::value;
      static_for<0, TN>([&](auto ii) {
        constexpr int i = decltype(ii)::value;
        acc[i][k] = mma<(i & 1) * 2 + ks, (k & 1) * 2 + ks>(cur.a[i], cur.b[k], acc[i][k], sc.a[i >> 1], sc.b[k >> 1]);
      });
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
  Scales sc, sn;
  constexpr std::integral_constant<int, 0> k0{};
  constexpr std::integral_constant<int, 1> k1{};
  static_for<0, NR>([&](auto q) { read1(f0, 0, k0, q); });
  read_scales(sc, 0);
  int slot = 0;
  for (int t = 0; t < nst; ++t) {
    const int next = slot + 1 == NS ? 0 : slot + 1;
    phase(f0, sc, f1, slot, k1, 0, std::false_type{});
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NS - 2) * LPS) : "memory");
    read_scales(sn, next);
    phase(f1, sc, f0, next, k0, slot, std::true_type{});
    sc = sn;
    ++issued;
    slot = next;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  // Epilogue: lane = row of each row tile, 8 consecutive channels per pair of channel tiles; the
  // residuals of a batch of rows are on their way together
  const ActClamp ac = act_clamp_of(p.act, p.alpha);
  constexpr int BATCH = F32 ? 1 : TM;
  auto row_of = [&](int k) { return m0 + wrow + (k >> 1) * 32 + (k & 1) * 4 + prow; };
  auto epilogue = [&](auto mode_tag) {
#pragma unroll
    for (int pr = 0; pr < TN / 2; ++pr) {
      const int n = n0 + wn * WTN + pr * 32 + lc * 8;
      if (n >= p.N) continue;
      float bias[8];
      if (p.bias) {
        load8f(p.bias + n, bias);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[e] = 0.0f;
      }
#pragma unroll
      for (int kb = 0; kb < TM; kb += BATCH) {
        Chunk<F32> res[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) res[k] = load_res<F32>(p, min(row_of(kb + k), p.M - 1), n);
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
          const int m = row_of(kb + k);
          if (m >= p.M) continue;
          float a[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] = acc[2 * pr + (e >> 2)][kb + k][e & 3];
          finish8<F32, decltype(mode_tag)::value>(p, a, bias, res[k], m, n, ac);
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

// Few rows: a workgroup of 8 waves owns 16 channels and all rows and splits the reduction over its waves, a
// stage of 256 codes each in turn, operands straight to registers, the waves' sums joined in LDS in their
// order; the time is that of reading the weights.  MT tiles of 16 rows.
//
// FUSED: the rows are quantized by every workgroup for itself, into LDS, while its first weights are on their
// way; that saves the launch that would do it.
constexpr int kRowWaves = 8;
constexpr int kRowThreads = 64 * kRowWaves;
constexpr int kRowStages = 2;  // stages per wave with loads in flight together
constexpr int kFusedCodes = 16 * kRowThreads;  // codes of all rows that FUSED takes

template <int MT, bool F32, bool FUSED>
__global__ __launch_bounds__(kRowThreads) void mxdense_rows_kernel(MxDenseParams p, MxRowsParams q) {
  __shared__ f32x4 red[kRowWaves][MT][64];
  __shared__ __align__(16) uint8_t codes[FUSED ? kFusedCodes / 2 : 16];
  __shared__ __align__(4) uint8_t scales[FUSED ? kFusedCodes / 32 : 4];  // [row][stage][block % 4][step]
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lc = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16;
  const int nst = p.Kq / kStageK, rb = p.Kq / 2;
  const uint8_t* wp = p.w + (int64_t)(n0 + lr) * rb + lc * 16;
  const uint8_t* wsp = p.ws + mx_scale_at(n0 + lr, lc, p.Kq);
  uint4 a[kRowStages][2];
  uint32_t as[kRowStages];
  auto load_w = [&](int t0) {
#pragma unroll
    for (int u = 0; u < kRowStages; ++u) {
      const int t = t0 + u * kRowWaves;
      const bool live = t < nst;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
        a[u][ks] = live ? *(const uint4*)(wp + (int64_t)t * 128 + ks * 64) : make_uint4(0u, 0u, 0u, 0u);
      as[u] = live ? *(const uint16_t*)(wsp + (int64_t)t * 256) : 0u;
    }
  };
  // this thread's 8 outputs, and what they need besides the sums: on its way from the start
  static_assert(MT * 32 <= kRowThreads, "an output group each");
  const int om = tid / 2, og = tid % 2, on = n0 + og * 8;
  const bool out = om < p.M && on < p.N && tid < MT * 32;
  float bias[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  Chunk<F32> res;
  load_w(wave);
  if (out) {
    if (p.bias) load8f(p.bias + on, bias);
    res = load_res<F32>(p, om, on);
  }
  if constexpr (FUSED) {
    const int chunks = p.Kq / 8, all = chunks * p.M;  // (32 chunks a stage: 4 lanes share a block)
    for (int i = tid; i < all; i += kRowThreads) {
      const int row = i / chunks, c = i - row * chunks;
      Chunk<F32> v;
      v.load(q.x, (int64_t)row * q.ldx, c * 8, q.K);
      const uint32_t byte = scale_byte(quad_max(top_bits(v)));
      *(uint32_t*)(codes + row * rb + c * 4) = codes_of(v, scale_power(byte));
      const int blk = c >> 2;
      if ((c & 3) == 0) scales[(row * nst + (blk >> 3)) * 8 + (blk & 3) * 2 + (blk >> 2 & 1)] = (uint8_t)byte;
    }
    __syncthreads();
  }
  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int t0 = wave; t0 < nst; t0 += kRowStages * kRowWaves) {
    uint4 b[kRowStages][MT][2];
    uint32_t bs[kRowStages][MT];
#pragma unroll
    for (int u = 0; u < kRowStages; ++u) {
      const int t = t0 + u * kRowWaves;
#pragma unroll
      for (int k = 0; k < MT; ++k) {
        const int m = k * 16 + lr;
        const bool live = m < p.M && t < nst;
        const uint8_t* xp = (FUSED ? codes : p.x) + (int64_t)m * rb + t * 128 + lc * 16;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) b[u][k][ks] = live ? *(const uint4*)(xp + ks * 64) : make_uint4(0u, 0u, 0u, 0u);
        const uint8_t* sp = FUSED ? scales + (m * nst + t) * 8 + lc * 2 : p.xs + mx_scale_at(m, lc, p.Kq) + (int64_t)t * 256;
        bs[u][k] = live ? *(const uint16_t*)sp : 0u;
      }
    }
    uint4 w[kRowStages][2];
    uint32_t wsc[kRowStages];
#pragma unroll
    for (int u = 0; u < kRowStages; ++u) {
      w[u][0] = a[u][0], w[u][1] = a[u][1];
      wsc[u] = as[u];
    }
    load_w(t0 + kRowStages * kRowWaves);
#pragma unroll
    for (int u = 0; u < kRowStages; ++u)
#pragma unroll
      for (int k = 0; k < MT; ++k) {
        acc[k] = mma<0, 0>(w[u][0], b[u][k][0], acc[k], wsc[u], bs[u][k]);
        acc[k] = mma<1, 1>(w[u][1], b[u][k][1], acc[k], wsc[u], bs[u][k]);
      }
  }
#pragma unroll
  for (int k = 0; k < MT; ++k) red[wave][k][lane] = acc[k];
  __syncthreads();
  // row m, channels n0 + 4 c .. + 3 sit in lane 16 c + m % 16 of tile m / 16 of every wave
  if (!out) return;
  const ActClamp ac = act_clamp_of(p.act, p.alpha);
  float sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const f32x4 r = red[w][om >> 4][(og * 2 + half) * 16 + (om & 15)];
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[4 * half + e] += r[e];
    }
  auto epilogue = [&](auto mode_tag) { finish8<F32, decltype(mode_tag)::value>(p, sum, bias, res, om, on, ac); };
  if (act_mode(p.act) == 1)
    epilogue(std::integral_constant<int, 1>{});
  else if (act_mode(p.act) == 0)
    epilogue(std::integral_constant<int, 0>{});
  else
    epilogue(std::integral_constant<int, 2>{});
}

template <bool F32>
hipError_t launch_rows(const MxDenseParams& p, const MxRowsParams& q, bool fused, hipStream_t s) {
  const int mt = (p.M + 15) / 16, grid = (p.N + 15) / 16;
  if (fused) mxdense_rows_kernel<1, F32, true><<<grid, kRowThreads, 0, s>>>(p, q);
  else if (mt == 1) mxdense_rows_kernel<1, F32, false><<<grid, kRowThreads, 0, s>>>(p, q);
  else if (mt == 2) mxdense_rows_kernel<2, F32, false><<<grid, kRowThreads, 0, s>>>(p, q);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

template <int BM, int BN, int WM, int WN, int NS, bool F32>
hipError_t launch_one(MxDenseParams p, hipStream_t s) {
  // the split of the tile grid over the XCDs that has each fetch the fewest operand rows
  const int ntm = (p.M + BM - 1) / BM, ntn = (p.N + BN - 1) / BN;
  int64_t best = INT64_MAX, blocks = 0;
  for (int py = 1; py <= 8; py *= 2) {
    const int mh = (ntm + 8 / py - 1) / (8 / py), nh = (ntn + py - 1) / py;
    const int64_t cost = (int64_t)mh * nh * 4096 + mh * BM + nh * BN;  // (first of all no XCD with more tiles)
    if (cost < best) best = cost, p.py = py, blocks = 8 * (int64_t)mh * nh;
  }
  mxdense_kernel<BM, BN, WM, WN, NS, F32><<<(unsigned)blocks, 64 * WM * WN, 0, s>>>(p);
  return hipGetLastError();
}

// Tiles (BM, BN, waves along each, ring stages) and what they cost in microseconds: a stage of 256 codes while
// at most one workgroup runs per CU or all slots (occ per CU) are busy, and a round's prologue and epilogue.
//   id BM BN WM WN NS  occ  lone  busy  round
#define BYOC_MXDENSE_TILES(X)                \
  X(0, 256, 256, 2, 4, 2, 1, 1.33, 1.8, 9.0) \
  X(1, 256, 128, 4, 2, 3, 1, 0.77, 1.0, 6.0) \
  X(2, 128, 128, 2, 4, 3, 1, 0.51, 0.6, 4.2) \
  X(3, 128, 128, 2, 4, 2, 2, 0.71, 1.09, 5.0) \
  X(4, 128, 64, 4, 2, 3, 2, 0.39, 0.70, 3.5) \
  X(5, 64, 64, 2, 2, 4, 2, 0.33, 0.46, 2.3)  \
  X(6, 32, 32, 2, 1, 8, 2, 0.26, 0.30, 1.8)

double tile_cost(int bm, int bn, int occ, double lone, double busy, double round, int64_t M, int64_t N, int64_t Kq) {
  const int64_t tiles = ((M + bm - 1) / bm) * ((N + bn - 1) / bn), slots = 256 * occ;
  const double stages = (double)(Kq / kStageK);
  const int64_t rest = tiles % slots;
  double t = (double)(tiles / slots) * (stages * busy + round);
  if (rest) t += stages * (rest <= (occ == 1 ? 128 : 256) ? lone : busy) + round;
  return t;
}

constexpr int kRowsN = 16 * 256;  // channels of the rows kernel: a workgroup of 16 for each CU

}  // namespace

hipError_t launch_mx_rows(const MxRowsParams& p, hipStream_t s) {
  if (p.rows < 1 || p.rows % 32 != 0 || p.Kq % kStageK != 0 || p.K > p.Kq) return hipErrorInvalidValue;
  const int64_t grid = (int64_t)(p.rows / 32) * (p.Kq / kStageK);
  if (p.f32) mx_rows_kernel<true><<<(unsigned)grid, 256, 0, s>>>(p);
  else mx_rows_kernel<false><<<(unsigned)grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

bool mxdense_fuses_rows(int64_t M, int64_t N, int64_t Kq) { return M <= 16 && M * Kq <= kFusedCodes && N <= kRowsN; }

hipError_t launch_mxdense_fused(const MxDenseParams& p, const MxRowsParams& q, hipStream_t s) {
  if (!mxdense_fuses_rows(p.M, p.N, p.Kq)) return hipErrorInvalidValue;
  return p.f32 ? launch_rows<true>(p, q, true, s) : launch_rows<false>(p, q, true, s);
}

MxDenseTile choose_mxdense_tile(int64_t M, int64_t N, int64_t Kq) {
  if (M <= 32 && N <= kRowsN) return {kMxDenseRows, (int)(M + 15) / 16 * 16, 16, 0};
  MxDenseTile best{};
  double least = INFINITY;
#define X(ID, BM, BN, WM, WN, NS, OCC, LONE, BUSY, ROUND)                                                \
  if (const double c = tile_cost(BM, BN, OCC, LONE, BUSY, ROUND, M, N, Kq); c < least) least = c, best = {ID, BM, BN, NS};
  BYOC_MXDENSE_TILES(X)
#undef X
  return best;
}

bool mxdense_tile_of(int id, MxDenseTile* t) {
#define X(ID, BM, BN, WM, WN, NS, OCC, LONE, BUSY, ROUND) \
  if (id == ID) return *t = {ID, BM, BN, NS}, true;
  BYOC_MXDENSE_TILES(X)
#undef X
  return false;
}

hipError_t launch_mxdense(const MxDenseParams& p, MxDenseTile t, hipStream_t s) {
  if (t.id == kMxDenseRows) return p.f32 ? launch_rows<true>(p, {}, false, s) : launch_rows<false>(p, {}, false, s);
#define X(ID, BM, BN, WM, WN, NS, OCC, LONE, BUSY, ROUND) \
  if (t.id == ID) return p.f32 ? launch_one<BM, BN, WM, WN, NS, true>(p, s) : launch_one<BM, BN, WM, WN, NS, false>(p, s);
  BYOC_MXDENSE_TILES(X)
#undef X
  return hipErrorInvalidValue;
}

}  // namespace byoc
