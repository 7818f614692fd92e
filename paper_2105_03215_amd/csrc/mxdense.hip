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
#include <climits>
#include <cmath>
#include <type_traits>

#include "dense_epilogue.h"
#include "lds_dma.h"

namespace byoc {
namespace {

using namespace dma;

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kStep = 128;  // codes along the reduction of a matrix instruction

// Codes and scales are kept in the order that the matrix instructions' lanes take them in: a block of 16 rows and
// a step of 128 codes is 1 KB, lane l's 16 bytes those of row l % 16 and of the 32 codes l / 16, which share a
// scale; it is moved to LDS and from there to registers without a calculated address or a bank conflict.  The blocks of a
// step follow one another, then those of the next step: workgroups that multiply different rows of a weight are at about the
// same step, and so read one stretch of memory together instead of places a power of two apart.
//
// Row r of a tensor is row r % 16 of block r / 16; of a weight that the tiles multiply (CHANNELS) the two
// blocks of 32 rows hold rows 8 (l / 4) + l % 4 and those 4 further on, so that a lane of the result has 8
// consecutive channels.
enum Order { ROWS = 0, CHANNELS = 1, ALONE = 2 };
struct Place {
  int block, lane;
};
__device__ __forceinline__ Place place_of(int r, int order) {
  if (order != CHANNELS) return Place{r >> 4, r & 15};
  return Place{(r >> 5) * 2 + (r >> 2 & 1), (r >> 3 & 3) * 4 + (r & 3)};
}
// Scales: a word for each lane, of four blocks in a row and one step; of a weight that the few-row kernel multiplies
// (ALONE, in the order of rows) of one block and four steps in a row.

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

// 64 rows x a step of 128 codes per workgroup (ALONE: 16 rows x 4 steps), 4 lanes of 8 values to a block of 32;
// the 4 KB of codes and 256 bytes of scales leave through LDS as they lie in memory.
template <bool F32>
__global__ __launch_bounds__(256) void mx_rows_kernel(MxRowsParams p) {
  __shared__ __align__(16) uint32_t codes[1024];
  __shared__ uint32_t words[64];
  const int tid = threadIdx.x, steps = p.Kq / kStep;
  const bool alone = p.order == ALONE;
  const int across = alone ? (steps + 3) / 4 : steps;
  const int g = blockIdx.x / across, a = blockIdx.x - g * across;
  const int row0 = g * (alone ? 16 : 64), step0 = a * (alone ? 4 : 1);
  // pass i: 16 rows of a step (ALONE: the i-th step of the rows)
  const int c = tid & 15;
  Chunk<F32> v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = row0 + (alone ? 0 : i * 16) + (tid >> 4), col = (step0 + (alone ? i : 0)) * kStep + c * 8;
    v[i].load(p.x, (int64_t)row * p.ldx, col, row < p.M ? p.K : 0);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const Place at = place_of((alone ? 0 : i * 16) + (tid >> 4), p.order);
    const int block = alone ? i : at.block, lane = (c >> 2) * 16 + at.lane;
    const uint32_t byte = scale_byte(quad_max(top_bits(v[i])));
    codes[(block * 64 + lane) * 4 + (c & 3)] = codes_of(v[i], scale_power(byte));
    if ((c & 3) == 0) ((uint8_t*)words)[lane * 4 + block] = (uint8_t)byte;
  }
  __syncthreads();
  const int block = tid >> 6, lane = tid & 63;
  const int blocks = p.rows / 16;
  const int64_t at = alone ? (int64_t)(step0 + block) * blocks + g : (int64_t)a * blocks + g * 4 + block;
  if (!alone || step0 + block < steps) ((uint4*)p.q)[at * 64 + lane] = ((const uint4*)codes)[tid];
  if (tid < 64) ((uint32_t*)p.scale)[((int64_t)a * (alone ? blocks : blocks / 4) + g) * 64 + tid] = words[tid];
}

// D += A B of 128 codes, each with the scale byte SA / SB of its lane's word.
template <int SA, int SB>
__device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c, uint32_t sa, uint32_t sb) {
  const i32x8 a8 = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  const i32x8 b8 = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, SA, (int)sa, SB, (int)sb);
}

// A block (16 bytes per lane) or a word per lane from a buffer straight into LDS, `at` bytes on (as lds_fill16).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void fill_block(i32x4 rsrc, uint32_t lds_addr, uint32_t voff, int at) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(lds_addr), "v"(voff), "s"(rsrc), "s"(at)
               : "memory", "m0");
}
__device__ __forceinline__ void fill_words(i32x4 rsrc, uint32_t lds_addr, uint32_t voff, int at) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, %3 offen lds"
               :
               : "s"(lds_addr), "v"(voff), "s"(rsrc), "s"(at)
               : "memory", "m0");
}
#pragma clang diagnostic pop

constexpr int kNoAct = 4;  // of an epilogue without an activation (its others are act_apply's)

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
// HBM -> LDS through a ring of NS stages of KS steps of 128 codes, with one barrier a stage, the MFMA operands of a
// step read while the previous step multiplies.
template <int BM, int BN, int WM, int WN, int KS, int NS, bool F32>
__global__ __launch_bounds__(64 * WM * WN) void mxdense_kernel(MxDenseParams p) {
  constexpr int NW = WM * WN;
  constexpr int WTM = BM / WM, WTN = BN / WN;
  constexpr int TM = WTM / 16, TN = WTN / 16;
  constexpr int GM = BM / 16, GN = BN / 16;                // blocks of a step
  constexpr int SM = (BM + 63) / 64, SN = (BN + 63) / 64;  // words of scales a lane
  constexpr int AR = GM * KS / NW, BR = GN * KS / NW, SR = ((SM + SN) * KS + NW - 1) / NW;  // of them a wave and stage
  static_assert(GM * KS % NW == 0 && GN * KS % NW == 0, "fill shape");
  static_assert(WTM % 16 == 0 && WTN % 32 == 0, "wave tile: whole MFMA rows, pairs of channel tiles");
  static_assert((TM % 4 == 0 || 4 % TM == 0) && (TN % 4 == 0 || 4 % TN == 0), "scales: whole words or a part of one");
  static_assert(KS == 2 || (KS == 1 && NS % 2 == 0), "turns of one step come in pairs");
  constexpr int LPS = AR + BR + SR;
  constexpr int CODES = (GM + GN) * KS * 64;    // uint4 per stage
  constexpr int STAGE = CODES + SR * NW * 16;   // with the scales
  static_assert(NS >= 2 && (NS - 1) * LPS <= 63, "vmcnt immediate");
  static_assert(NS * STAGE * 16 <= kLdsLimit, "LDS");
  __shared__ uint4 ring[NS * STAGE];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;

  // XCD x = (gx, gy) of 8 / py x py owns a block of the tile grid (workgroup b runs on XCD b % 8) and
  // walks it in bands of 4 row tiles; its workgroups take every gridDim / 8-th of them
  constexpr int kBand = 4;
  const int ntm = (p.M + BM - 1) / BM, ntn = (p.N + BN - 1) / BN;
  const int x = blockIdx.x & 7;
  const int px = 8 / p.py;
  const int mh = (ntm + px - 1) / px, nh = (ntn + p.py - 1) / p.py;
  const int gx = x / p.py, gy = x - gx * p.py;
  int j = blockIdx.x >> 3;
  struct Tile {
    int m0, n0;  // m0 < 0: none
  };
  auto next_tile = [&] {
    for (; j < mh * nh; j += gridDim.x >> 3) {
      const int band = j / (kBand * nh), at = j - band * kBand * nh;
      const int bm = min(kBand, mh - band * kBand), jn = at / bm;
      const int tm = gx * mh + band * kBand + at - jn * bm, tn = gy * nh + jn;
      if (tm >= ntm || tn >= ntn) continue;
      j += gridDim.x >> 3;
      return Tile{tm * BM, tn * BN};
    }
    return Tile{-1, 0};
  };
  const int steps = p.Kq / kStep, stages = steps / KS;

  // What this wave fills of a stage: blocks wave, wave + NW, ... of each operand, step by step, and words of scales.
  // (Blocks past the rows' last read what is there in their place: rows that are not used.)
  const int mb = (p.M + 63) / 64 * 4, nb = p.blocks;  // blocks of the rows and of the weight, of a step
  i32x4 xr, wr, sr[SR];
  int x_at[AR], w_at[BR], s_at[SR], s_step[SR];  // bytes from the tile's first stage to the blocks and words of this wave's
  auto set_tile = [&](Tile t) {
    constexpr int kAll = 0x7FFFFFFF;
    xr = buffer_rsrc(p.x + (int64_t)(t.m0 / 16) * 1024, kAll);
    wr = buffer_rsrc(p.w + (int64_t)(t.n0 / 16) * 1024, kAll);
#pragma unroll
    for (int i = 0; i < AR; ++i) {
      const int g = i * NW + wave;
      x_at[i] = (g / GM * mb + min(g % GM, mb - 1 - t.m0 / 16)) * 1024;
    }
#pragma unroll
    for (int i = 0; i < BR; ++i) {
      const int g = i * NW + wave;
      w_at[i] = (g / GN * nb + g % GN) * 1024;
    }
#pragma unroll
    for (int i = 0; i < SR; ++i) {
      const int g = min(i * NW + wave, (SM + SN) * KS - 1), of = g % (SM + SN);
      const bool rows = of < SM;
      sr[i] = buffer_rsrc(rows ? p.xs + (int64_t)min(t.m0 / 64 + of, mb / 4 - 1) * 256
                               : p.ws + (int64_t)(t.n0 / 64 + of - SM) * 256, kAll);
      s_step[i] = (rows ? mb : nb) / 4 * 256;
      s_at[i] = g / (SM + SN) * s_step[i];
    }
  };
  Tile tile = next_tile();
  if (tile.m0 < 0) return;
  set_tile(tile);
  const uint32_t off16 = lane * 16, off4 = lane * 4;
  // (Scalar instructions are not hidden where a SIMD has one wave: what can be is formed once, per wave or per stage.)
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(ring));
  uint32_t x_to[AR], w_to[BR];  // LDS places of the blocks in slot 0
#pragma unroll
  for (int i = 0; i < AR; ++i) {
    const int g = i * NW + wave;
    x_to[i] = __builtin_amdgcn_readfirstlane(lds0 + (g / GM * (GM + GN) + g % GM) * 1024);
  }
#pragma unroll
  for (int i = 0; i < BR; ++i) {
    const int g = i * NW + wave;
    w_to[i] = __builtin_amdgcn_readfirstlane(lds0 + (g / GN * (GM + GN) + GM + g % GN) * 1024);
  }
  int issued = 0;
  struct Fill {
    uint32_t slot;  // bytes of the slot
    int x, w, t;    // bytes of the stage's first step, and its number
  };
  auto next_fill = [&](int slot) {
    const int t = min(issued, stages - 1) * KS;  // (past the last stage: what is not used)
    ++issued;
    return Fill{(uint32_t)(slot * STAGE * 16), t * mb * 1024, t * nb * 1024, t};
  };
  auto fill = [&](const Fill& f, auto q_tag) {
    constexpr int q = decltype(q_tag)::value;
    if constexpr (q < AR)
      fill_block(xr, x_to[q] + f.slot, off16, x_at[q] + f.x);
    else if constexpr (q < AR + BR)
      fill_block(wr, w_to[q - AR] + f.slot, off16, w_at[q - AR] + f.w);
    else
      fill_words(sr[q - AR - BR], lds0 + CODES * 16 + ((q - AR - BR) * NW + wave) * 256 + f.slot, off4,
                 s_at[q - AR - BR] + f.t * s_step[q - AR - BR]);
  };

  f32x4 acc[TN][TM];
  const int lr = lane & 15, lc = lane >> 4;
  constexpr int PM = (TM + 3) / 4, PN = (TN + 3) / 4;
  struct Frags {
    uint4 a[TN], b[TM];
    uint32_t sa[PN], sb[PM];
  };
  constexpr int NR = TN + TM + PN + PM;
  auto read1 = [&](Frags& f, int slot, auto ks_tag, auto q_tag) {
    constexpr int q = decltype(q_tag)::value, ks = decltype(ks_tag)::value;
    const uint4* const st = ring + slot * STAGE + ks * (GM + GN) * 64 + lane;
    const uint32_t* const sc = (const uint32_t*)(ring + slot * STAGE + CODES) + ks * (SM + SN) * 64 + lane;
    if constexpr (q < PN)
      f.sa[q] = sc[(SM + wn * TN / 4 + q) * 64];
    else if constexpr (q < PN + PM)
      f.sb[q - PN] = sc[(wm * TM / 4 + q - PN) * 64];
    else if constexpr (q < PN + PM + TN)
      f.a[q - PN - PM] = st[(GM + wn * TN + q - PN - PM) * 64];
    else
      f.b[q - PN - PM - TN] = st[(wm * TM + q - PN - PM - TN) * 64];
  };
  int sa_at = 0, sb_at = 0;  // bits
  // The step in cur multiplies while step ks of a slot is read and, FILL, a slot filled.
  auto phase = [&](const Frags& cur, Frags& nxt, int rslot, auto ks_tag, const Fill& f, auto fill_tag) {
    constexpr int RG = TM > 4 ? TM - 2 : TM;
    // (a wave with less than four tiles has them at the place of its own in the word)
    uint32_t sa[PN], sb[PM];
#pragma unroll
    for (int i = 0; i < PN; ++i) sa[i] = TN < 4 ? cur.sa[i] >> sa_at : cur.sa[i];
#pragma unroll
    for (int i = 0; i < PM; ++i) sb[i] = TM < 4 ? cur.sb[i] >> sb_at : cur.sb[i];
    static_for<0, TM>([&](auto jj) {
      constexpr int k = decltype(jj)::value;
      static_for<0, TN>([&](auto ii) {
        constexpr int i = decltype(ii)::value;
        acc[i][k] = mma<i & 3, k & 3>(cur.a[i], cur.b[k], acc[i][k], sa[i >> 2], sb[k >> 2]);
      });
      static_for<0, NR>([&](auto q) {
        if constexpr (decltype(q)::value * RG / NR == k) read1(nxt, rslot, ks_tag, q);
      });
      if constexpr (decltype(fill_tag)::value)
        static_for<0, LPS>([&](auto q) {
          if constexpr (decltype(q)::value * TM / LPS == k) fill(f, q);
        });
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  static_for<0, NS>([&](auto i) {
    const Fill f = next_fill(decltype(i)::value);
    static_for<0, LPS>([&](auto q) { fill(f, q); });
  });
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((NS - 1) * LPS) : "memory");
  Frags f0, f1;
  int slot = 0;
  constexpr std::integral_constant<int, 0> k0{};
  constexpr std::integral_constant<int, 1> k1{};
  // A stage's last step is in registers, read by every wave before the barrier: its slot takes the stage NS
  // further on, while the next stage's first step, which has landed for every wave, is read.
  auto last_step = [&](const Frags& cur, Frags& nxt) {
    const int next = slot + 1 == NS ? 0 : slot + 1;
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NS - 2) * LPS) : "memory");
    phase(cur, nxt, next, k0, next_fill(slot), std::true_type{});
    slot = next;
  };
  auto turns = [&](int t, int end) {
    if constexpr (KS == 2) {
      for (; t < end; ++t) {
        phase(f0, f1, slot, k1, Fill{}, std::false_type{});
        last_step(f1, f0);
      }
    } else {
      for (; t < end; t += 2) {
        last_step(f0, f1);
        last_step(f1, f0);
      }
    }
  };
  const ActClamp ac = act_clamp_of(p.act, p.alpha);
  // Epilogue: lane = row of each row tile, 8 consecutive channels per pair of channel tiles.  With every check
  // it is bound by the vector ALU (at 4 cycles an instruction, 550 cycles for 8 values with a residual of zeros: 7.4 us a
  // tile of 256 x 256 beside the 25 us of a product over 4096), so that whole tiles without a residual or an activation
  // have forms of their own.
  constexpr int NP = TN / 2, BATCH = F32 ? 1 : TM * NP > 16 ? 16 / NP : TM;  // (rows whose residuals are on their way together)
  auto epilogue = [&](auto mode_tag, auto res_tag, auto whole_tag) {
    const int row0 = tile.m0 + wm * WTM + lr, col0 = tile.n0 + wn * WTN + lc * 8;
    constexpr int MODE = decltype(mode_tag)::value;
    constexpr bool RES = decltype(res_tag)::value, WHOLE = decltype(whole_tag)::value;
    float bias[NP][8];
#pragma unroll
    for (int pr = 0; pr < NP; ++pr) {
      if (p.bias) {
        load8f(p.bias + col0 + pr * 32, bias[pr]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[pr][e] = 0.0f;
      }
    }
#pragma unroll
    for (int kb = 0; kb < TM; kb += BATCH) {
      Chunk<F32> res[RES ? BATCH : 1][NP];
      if constexpr (RES) {
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
#pragma unroll
          for (int pr = 0; pr < NP; ++pr) {
            if constexpr (WHOLE) res[k][pr].load(p.res, (row0 + (kb + k) * 16) * p.ldr, col0 + pr * 32, INT_MAX);
            else res[k][pr] = load_res<F32>(p, min(row0 + (kb + k) * 16, p.M - 1), col0 + pr * 32);
          }
      }
#pragma unroll
      for (int k = 0; k < BATCH; ++k)
#pragma unroll
        for (int pr = 0; pr < NP; ++pr) {
          const int m = row0 + (kb + k) * 16, n = col0 + pr * 32;
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = acc[2 * pr + (e >> 2)][kb + k][e & 3] + bias[pr][e];
          if constexpr (RES) {
            float r[8];
            res[k][pr].get(r);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += r[e];
          }
          if constexpr (MODE != kNoAct) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = act_nan<F32, MODE>(v[e], ac);
          }
          if constexpr (WHOLE) store_chunk<F32>(p.y, m * p.ldy, n, INT_MAX, v);
          else if (m < p.M && n < p.N) store_chunk<F32>(p.y, m * p.ldy, n, p.N, v);
        }
    }
  };
  auto finish = [&](auto mode_tag) {
    const bool whole = tile.m0 + BM <= p.M && tile.n0 + BN <= min(p.N, p.channels);
    if (p.res) {
      if (whole) epilogue(mode_tag, std::true_type{}, std::true_type{});
      else epilogue(mode_tag, std::true_type{}, std::false_type{});
    } else {
      if (whole) epilogue(mode_tag, std::false_type{}, std::true_type{});
      else epilogue(mode_tag, std::false_type{}, std::false_type{});
    }
  };
  // The last turns of a tile fill the ring with the first steps of the next one, which land during the epilogue.
  for (;;) {
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int k = 0; k < TM; ++k) acc[i][k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    sa_at = 8 * ((wn * TN + tile.n0 / 16) % 4), sb_at = 8 * ((wm * TM + tile.m0 / 16) % 4);
    static_for<0, NR>([&](auto q) { read1(f0, slot, k0, q); });
    turns(0, stages - NS);
    const Tile next = next_tile();
    if (next.m0 >= 0) {
      set_tile(next);
      issued = 0;
    }
    turns(max(0, stages - NS), stages);
    if (p.act == kActNone)
      finish(std::integral_constant<int, kNoAct>{});
    else if (act_mode(p.act) == 1)
      finish(std::integral_constant<int, 1>{});
    else
      finish(std::integral_constant<int, 0>{});
    if (next.m0 < 0) break;
    tile = next;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// Few rows: a workgroup of 8 waves owns 16 channels and all rows and splits the reduction over its waves, a
// step of 128 codes each in turn, operands straight to registers, the waves' sums joined in LDS in their
// order; the time is that of reading the weights.  MT blocks of 16 rows.
//
// FUSED: the rows are quantized by every workgroup for itself, into LDS, while its first weights are on their
// way; that saves the launch that would do it.
constexpr int kRowWaves = 8;
constexpr int kRowThreads = 64 * kRowWaves;
constexpr int kRowSteps = 4;                   // steps per wave with loads in flight together
constexpr int kFusedCodes = 64 * kRowThreads;  // codes of all rows that FUSED takes

template <int MT, bool F32, bool FUSED>
__global__ __launch_bounds__(kRowThreads) void mxdense_rows_kernel(MxDenseParams p, MxRowsParams q) {
  __shared__ f32x4 red[kRowWaves][MT][64];
  __shared__ __align__(16) uint8_t codes[FUSED ? kFusedCodes / 2 : 16];  // [row][Kq / 2]
  __shared__ uint8_t scales[FUSED ? kFusedCodes / 32 : 4];               // [row][Kq / 32]
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lc = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16;
  const int steps = p.Kq / kStep;
  const uint4* const wp = (const uint4*)p.w + (int64_t)blockIdx.x * 64 + lane;
  const uint32_t* const wsp = (const uint32_t*)p.ws + (int64_t)blockIdx.x * 64 + lane;
  uint4 a[kRowSteps];
  uint32_t as[kRowSteps];
  auto load_w = [&](int t0) {
#pragma unroll
    for (int u = 0; u < kRowSteps; ++u) {
      const int t = t0 + u * kRowWaves;
      a[u] = t < steps ? wp[(int64_t)t * p.blocks * 64] : make_uint4(0u, 0u, 0u, 0u);
      as[u] = t < steps ? wsp[(int64_t)(t >> 2) * p.blocks * 64] >> (8 * (t & 3)) : 0u;
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
    const int chunks = p.Kq / 8, all = chunks * p.M;  // (16 chunks a step: 4 lanes share a block)
    for (int i = tid; i < all; i += kRowThreads) {
      const int row = i / chunks, c = i - row * chunks;
      Chunk<F32> v;
      v.load(q.x, (int64_t)row * q.ldx, c * 8, q.K);
      const uint32_t byte = scale_byte(quad_max(top_bits(v)));
      *(uint32_t*)(codes + row * (p.Kq / 2) + c * 4) = codes_of(v, scale_power(byte));
      if ((c & 3) == 0) scales[row * (p.Kq / 32) + (c >> 2)] = (uint8_t)byte;
    }
    __syncthreads();
  }
  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int t0 = wave; t0 < steps; t0 += kRowSteps * kRowWaves) {
    uint4 b[kRowSteps][MT];
    uint32_t bs[kRowSteps];
#pragma unroll
    for (int u = 0; u < kRowSteps; ++u) {
      const int t = t0 + u * kRowWaves;
      bs[u] = 0u;
#pragma unroll
      for (int k = 0; k < MT; ++k) b[u][k] = make_uint4(0u, 0u, 0u, 0u);
      if (t >= steps) continue;
      if constexpr (FUSED) {
        if (lr < p.M) {
          b[u][0] = *(const uint4*)(codes + lr * (p.Kq / 2) + t * 64 + lc * 16);
          bs[u] = scales[lr * (p.Kq / 32) + t * 4 + lc];
        }
      } else {
        bs[u] = ((const uint32_t*)p.xs)[t * 64 + lane];  // (up to 64 rows: one word, four blocks a step)
#pragma unroll
        for (int k = 0; k < MT; ++k) b[u][k] = ((const uint4*)p.x)[(t * 4 + k) * 64 + lane];
      }
    }
    uint4 w[kRowSteps];
    uint32_t wsc[kRowSteps];
#pragma unroll
    for (int u = 0; u < kRowSteps; ++u) w[u] = a[u], wsc[u] = as[u];
    load_w(t0 + kRowSteps * kRowWaves);
#pragma unroll
    for (int u = 0; u < kRowSteps; ++u)
      static_for<0, MT>([&](auto k) {
        constexpr int K = decltype(k)::value;
        acc[K] = mma<0, K>(w[u], b[u][K], acc[K], wsc[u], bs[u]);
      });
  }
#pragma unroll
  for (int k = 0; k < MT; ++k) red[wave][k][lane] = acc[k];
  __syncthreads();
  // row m, channels n0 + 4 c .. + 3 sit in lane 16 c + m % 16 of block m / 16 of every wave
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
  else if (mt == 3) mxdense_rows_kernel<3, F32, false><<<grid, kRowThreads, 0, s>>>(p, q);
  else if (mt == 4) mxdense_rows_kernel<4, F32, false><<<grid, kRowThreads, 0, s>>>(p, q);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

template <int BM, int BN, int WM, int WN, int KS, int NS, int OCC, bool F32>
hipError_t launch_one(MxDenseParams p, hipStream_t s) {
  // the split of the tile grid over the XCDs that has each fetch the fewest operand rows
  const int ntm = (p.M + BM - 1) / BM, ntn = (p.N + BN - 1) / BN;
  int64_t best = INT64_MAX, blocks = 0;
  for (int py = 1; py <= 8; py *= 2) {
    const int mh = (ntm + 8 / py - 1) / (8 / py), nh = (ntn + py - 1) / py;
    const int64_t cost = (int64_t)mh * nh * 4096 + mh * BM + nh * BN;  // (first of all no XCD with more tiles)
    if (cost < best) best = cost, p.py = py, blocks = 8 * (int64_t)mh * nh;
  }
  // (a reduction shorter than the ring leaves no room for the next tile in it: a workgroup for each)
  if (p.Kq >= NS * KS * kStep) blocks = std::min<int64_t>(blocks, 256 * OCC);
  mxdense_kernel<BM, BN, WM, WN, KS, NS, F32><<<(unsigned)blocks, 64 * WM * WN, 0, s>>>(p);
  return hipGetLastError();
}

// Tiles (BM, BN, waves along each, steps of a stage, ring stages) and what they cost in microseconds: a step of 128
// codes while at most one workgroup runs per CU or all slots (occ per CU) are busy, and a round's start and end.
// Fitted to 22 shapes from 1 x 8192 x 12288 to 8192 x 4096 x 8192; the choice is the fastest tile, or within 1% of it, on 20
// of them, and 6% behind 128x64 on 300 x 4096 x 4096 and 128 x 4096 x 12288 (13.6 us for 12.85, 13.8 for 13.0), where
// the model has the two alike.  8192 x 4096 x 8192 of random rows with its quantization: 151 us as 256x256, 172 as 256x128,
// 182 as 128x128 twice a CU; of that the product takes 135, four tiles in a row of 32 steps of 0.78 us each (0.52 is what the
// matrix instructions need without operands to wait for) and an end of 9 us, which all workgroups
// reach together: the matrix cores are busy for 58% of the cycles, at a clock of 1.7 GHz.  (256x128 twice a CU, with 4 waves of
// 128 x 64 each: 233 us, as the LDS and the L2 then feed 41 bytes a cycle.)
//   id BM BN WM WN KS NS  occ  lone  busy  round
#define BYOC_MXDENSE_TILES(X)                       \
  X(0, 256, 256, 2, 4, 1, 4, 1, 0.535, 0.681, 7.46)  \
  X(1, 256, 128, 4, 2, 2, 3, 1, 0.319, 0.360, 6.37)  \
  X(2, 128, 128, 2, 4, 2, 4, 1, 0.202, 0.203, 5.17)  \
  X(3, 128, 128, 2, 4, 2, 2, 2, 0.285, 0.443, 4.34)  \
  X(4, 128, 64, 4, 2, 2, 3, 2, 0.136, 0.217, 5.00)   \
  X(5, 64, 64, 2, 2, 2, 4, 2, 0.077, 0.160, 4.23)    \
  X(6, 32, 32, 2, 1, 2, 8, 2, 0.010, 0.071, 4.45)

double tile_cost(int bm, int bn, int occ, double lone, double busy, double round, int64_t M, int64_t N, int64_t Kq) {
  const int64_t tiles = ((M + bm - 1) / bm) * ((N + bn - 1) / bn), slots = 256 * occ;
  const double stages = (double)(Kq / kStep);
  const int64_t rest = tiles % slots;
  double t = (double)(tiles / slots) * (stages * busy + round);
  if (rest) t += stages * (rest <= (occ == 1 ? 128 : 256) ? lone : busy) + round;
  return t;
}

constexpr int64_t kRowsOutputs = 64 * 4096;  // rows (in blocks of 16) x channels that the rows kernel takes

}  // namespace

hipError_t launch_mx_rows(const MxRowsParams& p, hipStream_t s) {
  if (p.rows < 1 || p.rows % 64 != 0 || p.Kq % (2 * kStep) != 0 || p.K > p.Kq) return hipErrorInvalidValue;
  const int steps = p.Kq / kStep;
  const int64_t grid = p.order == ALONE ? (int64_t)(p.rows / 16) * ((steps + 3) / 4) : (int64_t)(p.rows / 64) * steps;
  if (p.f32) mx_rows_kernel<true><<<(unsigned)grid, 256, 0, s>>>(p);
  else mx_rows_kernel<false><<<(unsigned)grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

int64_t mx_code_bytes(int64_t rows, int64_t Kq) { return rows * Kq / 2; }
int64_t mx_scale_bytes(int64_t rows, int64_t Kq) { return (rows + 15) / 16 * ((Kq / kStep + 3) / 4 * 4) * 64; }
int mx_weight_order(MxDenseTile t) { return t.id == kMxDenseRows ? ALONE : CHANNELS; }

// (1 x 4096 x 4096: 5.0 us, 7.7 with a launch for the rows; 8 x 4096 x 4096, where every workgroup quantizes 32768
// values, 6.9 and 7.9; 1 x 8192 x 8192 9.1 and 11.9)
bool mxdense_fuses_rows(int64_t M, int64_t N, int64_t Kq) {
  return M <= 16 && M * Kq <= kFusedCodes && 16 * N <= kRowsOutputs;
}

hipError_t launch_mxdense_fused(const MxDenseParams& p, const MxRowsParams& q, hipStream_t s) {
  if (!mxdense_fuses_rows(p.M, p.N, p.Kq)) return hipErrorInvalidValue;
  return p.f32 ? launch_rows<true>(p, q, true, s) : launch_rows<false>(p, q, true, s);
}

// The rows kernel up to 64 rows, fewer the more channels there are (32 x 4096 x 4096: 7.5 us, 10.1 on 32x32 tiles; 64 x
// 4096 x 4096 7.8 and 10.1; 1 x 8192 x 8192 11.8 and 14.6; but 64 x 8192 x 8192, as every workgroup reads all rows,
// 17.1 and 15.5); else the tile of least modelled time.
MxDenseTile choose_mxdense_tile(int64_t M, int64_t N, int64_t Kq) {
  if (M <= 64 && (M + 15) / 16 * 16 * N <= kRowsOutputs) return {kMxDenseRows, (int)(M + 15) / 16 * 16, 16, 0};
  MxDenseTile best{};
  double least = INFINITY;
#define X(ID, BM, BN, WM, WN, KS, NS, OCC, LONE, BUSY, ROUND)                                                \
  if (const double c = tile_cost(BM, BN, OCC, LONE, BUSY, ROUND, M, N, Kq); c < least) least = c, best = {ID, BM, BN, NS};
  BYOC_MXDENSE_TILES(X)
#undef X
  return best;
}

bool mxdense_tile_of(int id, MxDenseTile* t) {
#define X(ID, BM, BN, WM, WN, KS, NS, OCC, LONE, BUSY, ROUND) \
  if (id == ID) return *t = {ID, BM, BN, NS}, true;
  BYOC_MXDENSE_TILES(X)
#undef X
  return false;
}

hipError_t launch_mxdense(const MxDenseParams& p, MxDenseTile t, hipStream_t s) {
  if (t.id == kMxDenseRows) return p.f32 ? launch_rows<true>(p, {}, false, s) : launch_rows<false>(p, {}, false, s);
#define X(ID, BM, BN, WM, WN, KS, NS, OCC, LONE, BUSY, ROUND) \
  if (t.id == ID) return p.f32 ? launch_one<BM, BN, WM, WN, KS, NS, OCC, true>(p, s) : launch_one<BM, BN, WM, WN, KS, NS, OCC, false>(p, s);
  BYOC_MXDENSE_TILES(X)
#undef X
  return hipErrorInvalidValue;
}

}  // namespace byoc
