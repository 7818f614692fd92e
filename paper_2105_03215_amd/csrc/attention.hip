// Softmax attention with keys of another length than the queries: cross
// attention to an encoder's states, causal self attention, single tokens over a
// long context.
//
// One pass over the keys with the running maximum and sum of the softmax:
//   m' = max(m, max_j s_j),  l' = l 2^(m - m') + sum_j 2^(s_j - m'),
//   o' = o 2^(m - m') + sum_j 2^(s_j - m') v_j,   o / l at the end,
// with s = (q . k) scale log2(e) in float32.
//
// Rows of queries are packed over the heads that share a key head: row
// r = i * group + g of (batch b, key head h) is query i of head h * group + g, so
// that one read of the keys serves the whole group.
//
// Both products run transposed on 32x32 MFMA tiles: S^T = K Q^T leaves 16 keys of
// one query row in each lane, so the softmax needs one exchange between the two
// halves of the wave, and its result is, in place, the right operand of
// O^T = V^T P^T: register group i of a lane half h holds keys 8 (i / 4) + 4 h + i % 4,
// and V^T is read in the same order (the order of a sum over keys is free).
#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

#include "lds_dma.h"

namespace byoc {
namespace {

using namespace dma;

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;

constexpr int kKeys = 32;   // keys of a tile
constexpr int kCols = 32;   // packed query rows of a tile
constexpr int kPitch = 33;  // of the waves' results in LDS: free of bank conflicts along either axis

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// max / sum over the two halves of the wave (lanes l and l ^ 32)
__device__ __forceinline__ float half_max(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Keys that packed row r of batch b sees.
__device__ __forceinline__ int seen_keys(const AttnParams& p, int len, int r) {
  if (r >= p.q_len * p.group) return 0;
  if (!p.causal) return len;
  return min(max(len - p.q_len + r / p.group + 1, 0), len);
}

// (a value that is the same in all lanes, said to the compiler: what is computed from it stays in scalar registers)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ int batch_len(const AttnParams& p, int b) {
  return p.lengths ? min(max(p.lengths[b], 0), p.k_len) : p.k_len;
}

// The key axis of few rows is split into p.chunks chunks, shared by the sequences in
// proportion to their lengths, which only the device knows: chunks of `size` tiles each,
// the first of sequence b number `first`, `count` of them, with the least size that needs
// no more than p.chunks.  That is at least ceil(tiles of all / chunks) and at most ceil(tiles
// of all / (chunks - batch)), as rounding up costs a sequence less than one chunk: each lane
// counts the chunks of one size between (16 x 1 over 16384 keys, 8 heads of 64: 146 us
// with the upper bound, which left half of the CUs without work, 114 so).
// More than 64 sequences (lanes) get the same number each.  chunks == batch: a sequence each.
// (floats of the workspace's head, a multiple of 4 so that the sums can be written 16 bytes at a time)
__host__ __device__ __forceinline__ int64_t head_floats(const AttnParams& p) { return (2 * (int64_t)p.batch + 3) / 4 * 4; }
struct Chunks {
  int first, count, size;
};
__device__ __forceinline__ Chunks lane_chunks(const AttnParams& p) {
  const int lane = threadIdx.x & 63;
  const int mine = lane < p.batch ? (batch_len(p, lane) + p.tile_keys - 1) / p.tile_keys : 0;
  int total = mine;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d, 64);
  Chunks c;
  const int spare = p.chunks - p.batch;
  const int low = max(1, (total + p.chunks - 1) / p.chunks), high = max(1, (total + spare - 1) / spare);
  const int size = low + lane * ((high - low + 62) / 63);
  const float inv = 1.0f / (float)size;
  int need = 0;
  for (int b = 0; b < p.batch; ++b) {
    const int n = __builtin_amdgcn_readlane(mine, b);
    int q = (int)((float)n * inv);  // (at most p.chunks: not more than 1 away from the quotient)
    const int r = n - q * size;
    q += r > size ? 2 : r > 0 ? 1 : r > -size ? 0 : -1;  // rounded up
    need += q;
  }
  const unsigned long long fits = __ballot(need <= p.chunks);
  c.size = __builtin_amdgcn_readlane(size, __builtin_ctzll(fits));  // (lane 63's is `high` or more: it fits)
  c.count = (mine + c.size - 1) / c.size;
  c.first = c.count;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int x = __shfl_up(c.first, d, 64);
    if (lane >= d) c.first += x;
  }
  c.first -= c.count;
  return c;
}
__device__ __forceinline__ Chunks uniform_chunks(const AttnParams& p, int b) {
  const int per = p.chunks / p.batch;
  const int tiles = (p.k_len + p.tile_keys - 1) / p.tile_keys;
  return Chunks{b * per, per, (tiles + per - 1) / per};
}
// The sequence of chunk q, -1 if no sequence needs it.
__device__ __forceinline__ int chunk_batch(const AttnParams& p, int q, Chunks* out) {
  if (p.batch > 64 || p.chunks == p.batch) {
    const int b = q / (p.chunks / p.batch);
    *out = uniform_chunks(p, b);
    return b;
  }
  const Chunks c = lane_chunks(p);
  const unsigned long long at = __ballot(q >= c.first && q < c.first + c.count);
  if (at == 0) return -1;
  const int b = __builtin_ctzll(at);
  *out = Chunks{__builtin_amdgcn_readlane(c.first, b), __builtin_amdgcn_readlane(c.count, b), uniform(c.size)};
  return b;
}
// The sequence with the n-th most keys (of at most 64; the lower number first among equals).
__device__ __forceinline__ int nth_longest(const AttnParams& p, int n) {
  const int lane = threadIdx.x & 63;
  const int mine = lane < p.batch ? batch_len(p, lane) : -1;
  int rank = 0;
  for (int j = 0; j < p.batch; ++j) {
    const int other = __builtin_amdgcn_readlane(mine, j);
    rank += other > mine || (other == mine && j < lane);
  }
  return __builtin_ctzll(__ballot(lane < p.batch && rank == n));
}
// The workspace: for each sequence the first of its chunks and their number (written by that chunk's
// workgroup, so that the join need not count them again; a sequence without keys has none), then the
// sums, then the maxima and weights.
__device__ __forceinline__ void note_chunks(const AttnParams& p, int b, int q, const Chunks& c) {
  if (q == c.first && threadIdx.x == 0) ((int2*)p.ws)[b] = make_int2(c.first, c.count);
}
// Where the result of chunk q of packed row `row` of key head kh stands: D sums, and its maximum and weight.
__device__ __forceinline__ float* part_sums(const AttnParams& p, int kh, int row, int q) {
  const int64_t rows = (int64_t)p.q_len * p.group;
  return p.ws + head_floats(p) + ((kh * rows + row) * p.chunks + q) * p.D;
}
__device__ __forceinline__ float* part_scale(const AttnParams& p, int kh, int row, int q) {
  const int64_t rows = (int64_t)p.q_len * p.group;
  return p.ws + head_floats(p) + (p.kv_heads * rows * p.D + (kh * rows + row) * 2) * p.chunks + q * 2;
}

// Swizzle keys of the LDS tiles, on 16-byte chunks of a row: key rows are read 16
// bytes per lane down the rows, value rows 8 bytes per lane with four rows and 16
// columns per 16 lanes; either way 16 lanes meet every bank once.
template <int CPR>
__device__ __forceinline__ int k_key(int row) {
  return CPR == 8 ? (row >> 1) & 7 : row & 15;
}
template <int CPR>
__device__ __forceinline__ int v_key(int row) {
  return CPR == 8 ? ((row >> 1) & 1) << 2 : ((row & 3) << 2) | ((row >> 2) & 3);
}

// Weights of 16 keys of one register group, rounded to bf16 for the matrix cores (a
// relative 2^-8 each at most, as the values' own rounding): an output is then 0.0021 of its size off instead of the
// 0.0016 of its own rounding.  Many rows take it, which are bound by the products: in two parts, as below,
// causal 2 x 4096, 32 heads over 8 of 128, is 360 us instead of 266, and 8 x 449 over up to 1027, 12 of 64, 23.7
// instead of 18.9.
__device__ __forceinline__ uint4 pack_weights(const f32x16& s, int ks) {
  return make_uint4(pack2_bf16(s[8 * ks + 0], s[8 * ks + 1]), pack2_bf16(s[8 * ks + 2], s[8 * ks + 3]),
                    pack2_bf16(s[8 * ks + 4], s[8 * ks + 5]), pack2_bf16(s[8 * ks + 6], s[8 * ks + 7]));
}

// The same in two parts, off by a relative 2^-16 together: the upper bits, and the rest rounded to bf16.  Few rows
// take it, whose time is that of the keys' and values' bytes (4 x 1 over up to 32768 keys, 32 heads over 8 of 128: 78 us
// either way; 16 x 1 over up to 1500, 12 of 64, where latency counts: 13.8 us, 13.0 with one part).  The
// rest is that of a weight 2^-20 larger, so that the parts of a weight above zero are both above zero (zero
// times an infinite value would be NaN).
__device__ __forceinline__ void pack_weights2(const f32x16& s, int ks, uint4* upper, uint4* rest) {
  uint32_t up[4], lo[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float w0 = s[8 * ks + 2 * e], w1 = s[8 * ks + 2 * e + 1];
    const float u0 = __uint_as_float(__float_as_uint(w0) & 0xFFFF0000u), u1 = __uint_as_float(__float_as_uint(w1) & 0xFFFF0000u);
    up[e] = __builtin_amdgcn_perm(__float_as_uint(w1), __float_as_uint(w0), 0x07060302u);
    lo[e] = pack2_bf16(__builtin_fmaf(w0, 1.0f + 0x1p-20f, -u0), __builtin_fmaf(w1, 1.0f + 0x1p-20f, -u1));
  }
  *upper = make_uint4(up[0], up[1], up[2], up[3]);
  *rest = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}

// V^T of 16 keys (row0 ..) and 32 columns (block d): the left operand of O^T = V^T P^T,
// keys in the order that pack_weights leaves them in.
template <int CPR>
__device__ __forceinline__ uint4 load_vt(const char* vt, int row0, int d, int lane) {
  const int h = lane >> 5;
  uint2 vf[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int r = row0 + 8 * j + 4 * h + ((lane & 15) >> 2);
    const int c = d * 4 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    const char* at = vt + r * (CPR * 16) + ((c ^ v_key<CPR>(r)) * 16) + (lane & 1) * 8;
    vf[j] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)at));
  }
  return make_uint4(vf[0].x, vf[0].y, vf[1].x, vf[1].y);
}

// Under a causal mask a wave's last tiles (two at most, as its rows' limits are less than 32 apart) hold keys that
// some of its rows do not see.  Their weights are zero, but zero times an infinite or NaN value is NaN: at the first
// of these tiles that holds one the wave stops, and add_keys adds the keys from there on one by one.  (1 x 4096, 32
// heads of 128: 156 us, up to 299 with a NaN; 1 x 1024, 8 heads of 64: 12 and 88; 2 x 2048, 8 heads of 256, where the
// check of 32 KB a tile counts most: 80.7 without it, 83.3.)
template <bool BF, int BYTES>
__device__ __forceinline__ bool holds_not_finite(const char* tile) {
  typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
  const uint4* at = (const uint4*)tile + (threadIdx.x & 63);
  uint32_t top = 0;
#pragma unroll 8
  for (int i = 0; i < BYTES / 1024; ++i) {
    const uint4 x = at[i * 64];
    for (uint32_t w : {x.x, x.y, x.z, x.w}) {
      if constexpr (BF)
        top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top),
                                                                     __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu)));
      else
        top = max(top, w & 0x7FFFFFFFu);
    }
  }
  return __any(BF ? max(top & 0xFFFFu, top >> 16) >= 0x7F80u : top >= 0x7F800000u);
}

// 4 columns of a row as floats.
__device__ __forceinline__ void load4(const bf16_t* p, float* v) {
  const uint2 u = *(const uint2*)p;
  v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xFFFF0000u);
  v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xFFFF0000u);
}
__device__ __forceinline__ void load4(const float* p, float* v) {
  const float4 u = *(const float4*)p;
  v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
}

// Adds keys j0 .. j1 - 1 to each row that sees them.
template <typename T, int DB, int QS>
__device__ __forceinline__ void add_keys(const AttnParams& p, const char* kb, const char* vb, int64_t sk, int64_t sv, int lim,
                                         int j0, int j1, const uint4* qf, float c2, f32x16* o, float& m, float& l) {
  constexpr int PER = 16 / sizeof(T);  // values of a 16-byte chunk
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll 1
  for (int j = j0; j < j1 && __any(j < lim); ++j) {
    const bool seen = j < lim;
    const T* const kr = (const T*)(kb + (int64_t)j * sk) + h * PER;
    const T* const vr = (const T*)(vb + (int64_t)j * sv) + 4 * h;
    float s = 0.0f;
#pragma unroll
    for (int st = 0; st < QS; ++st) {
      if (!seen || (2 * st + h) * PER >= p.D) continue;
      float a[8], b[8];
      const uint4 k = *(const uint4*)(kr + 2 * st * PER);
      if constexpr (PER == 8) {
        unpack8(k, a);
        unpack8(qf[st], b);
      } else {
        const f32x4 kf = __builtin_bit_cast(f32x4, k), qq = __builtin_bit_cast(f32x4, qf[st]);
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = kf[e], b[e] = qq[e];
      }
#pragma unroll
      for (int e = 0; e < PER; ++e) s = __builtin_fmaf(a[e], b[e], s);
    }
    s = half_sum(s) * c2;
    if (!seen) continue;
    const float mn = fmaxf(m, s), use = mn == -INFINITY ? 0.0f : mn;
    const float keep = exp2_(m - use), w = exp2_(s - use);
    m = mn;
    l = l * keep + (h == 0 ? w : 0.0f);  // (the halves' sums are added later)
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if (d * 32 + 8 * g + 4 * h >= p.D) continue;
        float v[4];
        load4(vr + d * 32 + 8 * g, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[d][4 * g + e] = o[d][4 * g + e] * keep + w * v[e];
      }
  }
}

// A workgroup takes 32 packed query rows of one (batch, key head) and a share of
// its keys; its waves take tiles of 32 keys in turn, each through its own LDS
// tiles, without a barrier until their results meet at the end.  Single tokens are
// bound by the keys' and values' bytes: 4 x 1 over up to 32768 keys, 32 heads over 8 of 128 (388 MB): 78 us,
// 5.0 TB/s.
//
// DP columns of a head in LDS (a power of two), DC of them multiplied.
template <typename T, int DP, int DC, int NW>
__global__ __launch_bounds__(64 * NW) void attention_rows_kernel(AttnParams p) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int ES = sizeof(T);
  constexpr int RB = DP * ES;         // bytes of an LDS row
  constexpr int CPR = RB / 16;        // its 16-byte chunks
  constexpr int TILE = kKeys * RB;    // bytes of a tile
  constexpr int NBUF = BF ? 2 : 1;
  constexpr int NI = TILE / 1024;     // loads of a tile per lane
  constexpr int DB = DC / 32;         // 32-column blocks of the output
  __shared__ __align__(16) char lds[NW * NBUF * 2 * TILE];
  __shared__ float ml[NW][2][kCols];
  static_assert(sizeof(lds) + sizeof(ml) <= kLdsLimit, "LDS");
  static_assert(NW * NBUF * 2 * TILE >= NW * DC * kPitch * 4, "the waves' results take the tiles' place");

  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, h = lane >> 5;
  const int wave = uniform(tid >> 6);
  const int R = p.q_len * p.group;
  const int ncb = (R + kCols - 1) / kCols;
  const int kh = blockIdx.x % p.kv_heads;
  const int rest = blockIdx.x / p.kv_heads;
  const int cb = ncb - 1 - rest % ncb, chunk = rest / ncb;  // (the last rows, which see the most keys, first)
  const bool joined = p.chunks > p.batch;
  Chunks ck;
  const int b = uniform(chunk_batch(p, chunk, &ck));
  if (b < 0) return;
  if (joined && cb == 0 && kh == 0) note_chunks(p, b, chunk, ck);
  const int len = uniform(batch_len(p, b));
  const int row = cb * kCols + col;
  const int lim = seen_keys(p, len, row);
  const int lim_lo = uniform(seen_keys(p, len, cb * kCols));  // (rows see more keys further down)
  const int kend = uniform(seen_keys(p, len, min(cb * kCols + kCols, R) - 1));
  const int t0 = (chunk - ck.first) * ck.size;
  const int t_end = min(t0 + ck.size, (kend + kKeys - 1) / kKeys);

  // this lane's part of its query row: 16-byte chunks 2 st + h
  constexpr int QS = DC * ES / 32;
  uint4 qf[QS];
  {
    const int i = row / p.group, g = row - i * p.group;
    const char* qp = (const char*)p.q + ((int64_t)(b * (int64_t)p.q_len + i) * p.ldq + (kh * p.group + g) * p.D) * ES;
#pragma unroll
    for (int st = 0; st < QS; ++st) {
      const int c = 2 * st + h;
      qf[st] = row < R && c * 16 < p.D * ES ? *(const uint4*)(qp + c * 16) : make_uint4(0u, 0u, 0u, 0u);
    }
  }

  const int64_t sk = p.ldk * ES, sv = p.ldv * ES;
  const char* kb = (const char*)p.k + (int64_t)b * p.k_len * sk + kh * p.D * ES;
  const char* vb = (const char*)p.v + (int64_t)b * p.k_len * sv + kh * p.D * ES;
  char* mine = lds + wave * (NBUF * 2 * TILE);
  // keys or values of a tile; rows past the length (and tiles past the end) read as zeros, whatever stands there
  auto fill = [&](int buf, int t, auto values_tag) {
    constexpr bool VALUES = decltype(values_tag)::value;
    const int k0 = t * kKeys;
    const int n = t < t_end ? min(kKeys, len - k0) : 0;
    const int64_t stride = VALUES ? sv : sk;
    const i32x4 r4 = buffer_rsrc((VALUES ? vb : kb) + (int64_t)k0 * stride, n > 0 ? (n - 1) * (int)stride + p.D * ES : 0);
    const uint32_t at = __builtin_amdgcn_readfirstlane(lds_addr(mine + (buf * 2 + VALUES) * TILE));
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int r = (i * 64 + lane) / CPR, s = (i * 64 + lane) % CPR;
      const int c = s ^ (VALUES ? v_key<CPR>(r) : k_key<CPR>(r));
      lds_fill16(r4, at + i * 1024, c * 16 < p.D * ES ? (uint32_t)(r * (int)stride + c * 16) : kOOB);
    }
  };
  constexpr std::integral_constant<bool, false> keys{};
  constexpr std::integral_constant<bool, true> values{};

  // LDS offsets of this lane's operands in a tile: its key row at chunk h, whose other chunks are an XOR away; and
  // (fp32) column col of value rows 4 h and on, where v_key(r + 4 h) = v_key(r) ^ h
  const uint32_t ka = col * RB + ((h ^ k_key<CPR>(col)) << 4);
  const uint32_t va = 4 * h * RB + (((col >> 2) ^ h) << 4) + (col & 3) * 4;

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = f32x16{};
  float m = -INFINITY, l = 0.0f;
  const float c2 = p.scale * 1.44269504088896340736f;
  const int masked = p.causal && p.q_len > 1 ? lim_lo / kKeys : INT_MAX;  // the first tile that some rows see a part of

  // Loads of 2 NBUF half tiles are in flight: a half is filled again as soon as it has been read.
  auto landed = [] { asm volatile("s_waitcnt vmcnt(%0)" ::"n"((2 * NBUF - 1) * NI) : "memory"); };
  auto read = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
  auto compute = [&](int buf, int t) {
    const char* kt = mine + buf * 2 * TILE;
    const char* vt = kt + TILE;
    landed();
    f32x16 s{};
#pragma unroll
    for (int st = 0; st < QS; ++st) {
      const uint4 a = *(const uint4*)(kt + (ka ^ (st % 8 << 5)) + st / 8 * 256);
      if constexpr (BF) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(qf[st]), s, 0, 0, 0);
      } else {
        const f32x4 af = __builtin_bit_cast(f32x4, a), bf = __builtin_bit_cast(f32x4, qf[st]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(af[e], bf[e], s, 0, 0, 0);
      }
    }
    read();
    fill(buf, t + NBUF * NW, keys);
    const int k0 = t * kKeys + 4 * h;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = k0 + 8 * (i >> 2) + (i & 3) < lim ? s[i] * c2 : -INFINITY;
      top = fmaxf(top, s[i]);
    }
    const float mn = fmaxf(m, half_max(top));
    const float use = mn == -INFINITY ? 0.0f : mn;  // (no key seen yet: every weight is zero)
    const float keep = exp2_(m - use);
    m = mn;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = exp2_(s[i] - use);
      sum += s[i];
    }
    l = l * keep + sum;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] *= keep;
    landed();
    if constexpr (BF) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        uint4 upper, rest, v[DB];
#pragma unroll
        for (int d = 0; d < DB; ++d) v[d] = load_vt<CPR>(vt, ks * 16, d, lane);
        pack_weights2(s, ks, &upper, &rest);
#pragma unroll
        for (int d = 0; d < DB; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v[d]), as_bf16x8(upper), o[d], 0, 0, 0);
#pragma unroll
        for (int d = 0; d < DB; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v[d]), as_bf16x8(rest), o[d], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = 8 * (i >> 2) + (i & 3);  // (and 4 h)
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const float vf = *(const float*)(vt + (va ^ ((v_key<CPR>(r) & 7) << 4)) + r * RB + ((d ^ (v_key<CPR>(r) >> 3)) * 128));
          o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[i], o[d], 0, 0, 0);
        }
      }
    }
  };

#pragma unroll
  for (int n = 0; n < NBUF; ++n) {
    fill(n, t0 + wave + n * NW, keys);
    fill(n, t0 + wave + n * NW, values);
  }
  int buf = 0, t = t0 + wave;
  for (; t < t_end; t += NW) {
    if (t >= masked) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((2 * NBUF - 2) * NI) : "memory");  // the tile's keys and values
      if (holds_not_finite<BF, TILE>(mine + (buf * 2 + 1) * TILE)) break;
    }
    compute(buf, t);
    read();
    fill(buf, t + NBUF * NW, values);
    buf = NBUF == 2 ? buf ^ 1 : 0;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  for (; t < t_end; t += NW) add_keys<T, DB, QS>(p, kb, vb, sk, sv, lim, t * kKeys, (t + 1) * kKeys, qf, c2, o, m, l);

  // the waves' results: a common maximum, then the sums in wave order
  l = half_sum(l);
  if (h == 0) {
    ml[wave][0][col] = m;
    ml[wave][1][col] = l;
  }
  __syncthreads();
  float top = ml[0][0][col];
#pragma unroll
  for (int w = 1; w < NW; ++w) top = fmaxf(top, ml[w][0][col]);
  const float use = top == -INFINITY ? 0.0f : top;
  const float f = exp2_(m - use);
  float* const os = (float*)lds;  // [wave][column][packed row]
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) os[(wave * DC + d * 32 + 8 * (i >> 2) + 4 * h + (i & 3)) * kPitch + col] = o[d][i] * f;
  float total = 0.0f;
#pragma unroll
  for (int w = 0; w < NW; ++w) total += ml[w][1][col] * exp2_(ml[w][0][col] - use);
  __syncthreads();
  if (wave == 0 && h == 0) {
    // the joined weight, where the outputs' threads find it; a row without keys is zero, one whose
    // seen scores are all -inf divides zero by zero, as the softmax does
    if (!joined) ml[0][1][col] = total;
    else if (row < R) {
      float* out = part_scale(p, kh, row, chunk);
      out[0] = top;
      out[1] = total;
    }
  }
  if (!joined) __syncthreads();
  // thread = 4 columns of a packed row, rows in turn
  const int rows = min(kCols, R - cb * kCols);
  for (int at = tid; at < rows * (DC / 4); at += 64 * NW) {
    const int c = at / (DC / 4), e = at % (DC / 4) * 4;
    if (e >= p.D) continue;
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = os[(e + j) * kPitch + c];
#pragma unroll
      for (int w = 1; w < NW; ++w) v[j] += os[(w * DC + e + j) * kPitch + c];
    }
    const int r = cb * kCols + c;
    if (joined) {
      *(float4*)(part_sums(p, kh, r, chunk) + e) = make_float4(v[0], v[1], v[2], v[3]);
      continue;
    }
    const float sum = ml[0][1][c];
    const bool any = seen_keys(p, len, r) > 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = any ? v[j] / sum : 0.0f;
    const int i = r / p.group, g = r - i * p.group;
    T* out = (T*)p.y + (b * (int64_t)p.q_len + i) * p.ldy + (kh * p.group + g) * p.D + e;
    if constexpr (BF) {
      *(uint2*)out = make_uint2(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]));
    } else {
      *(float4*)out = make_float4(v[0], v[1], v[2], v[3]);
    }
  }
}

// What a workgroup of `rows` packed rows works on.
struct Place {
  int b, kh, chunk, tile;  // b < 0: nothing
  Chunks ck;
};
__device__ __forceinline__ Place place(const AttnParams& p, int rows) {
  const int nh = p.chunks * p.kv_heads;
  const int nt = (p.q_len * p.group + rows - 1) / rows;
  Place w;
  if (p.lengths && !p.causal && p.chunks == p.batch && p.batch <= 64) {
    // sequences of different lengths: the longest first, all of its rows
    const int per = p.kv_heads * nt, pos = blockIdx.x / per, rem = blockIdx.x - pos * per;
    w.tile = rem / p.kv_heads;
    w.kh = rem - w.tile * p.kv_heads;
    w.b = w.chunk = uniform(nth_longest(p, pos));
    w.ck = uniform_chunks(p, w.b);
    return w;
  }
  // Head fastest: with a multiple of 8 heads each XCD (workgroup b runs on XCD b % 8) keeps to its own
  // heads' keys and values; the last rows first, which see the most keys under a causal mask.
  const int bh = blockIdx.x % nh;
  w.tile = nt - 1 - blockIdx.x / nh;
  w.chunk = bh / p.kv_heads;
  w.kh = bh - w.chunk * p.kv_heads;
  w.b = uniform(chunk_batch(p, w.chunk, &w.ck));
  return w;
}

// Many rows, bf16: four waves of 32 packed rows each share tiles of 64 keys and
// values, double-buffered in LDS; a tile's loads run while the one before is
// multiplied, with one barrier a tile.  Two such workgroups fit a CU (D <= 128), so
// that one's softmax runs beside the other's products.  Bound by both at 128 columns (causal 2 x 4096, 32 heads over 8
// of 128: 264 to 276 us, 1000 to 1040 TFLOP/s, the matrix cores busy for 58% of the cycles and the vector ALU for 56%), by the vector
// ALU at 64 (causal 2 x 4096, 12 of 64: 72 to 74 us, 39% and 65%); of sequences of different lengths by the longest one's chain
// of tiles (8 x 449 over 53 to 1027, 12 of 64: 19 us, 17 tiles in a row; 18% and 37%).
//
// The running maximum moves only when a tile's exceeds it by more than 2^8 (kSlack):
// the weights then stay under 2^8, far from overflow, and the 16 x D / 32 products
// that rescale the output are left out of almost every tile.
constexpr int kTileKeys = 64;
constexpr float kSlack = 8.0f;

//
// DP columns of a head in LDS (a power of two), DC of them multiplied (causal 2 x 2048, 20 heads over 4 of 80:
// 48.7 us with all 128, 43.2 with 96).
template <int DP, int DC, int KS>
__global__ __launch_bounds__(256, DP * KS <= 128 ? 2 : 1) void attention_tiles_kernel(AttnParams p) {
  constexpr int NW = 4 / KS;  // waves along the rows
  constexpr int RB = DP * 2, CPR = RB / 16;
  constexpr int TILE = kTileKeys * RB;
  constexpr int NI = TILE / (NW * 1024);  // loads of a tile per lane
  constexpr int DB = DC / 32, QS = DC / 16, KB = kTileKeys / 32;
  static_assert(DC % 32 == 0 && DC <= DP, "columns multiplied");
  __shared__ __align__(1024) char lds[KS * 4 * TILE];
  static_assert(sizeof(lds) <= kLdsLimit, "LDS");

  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, h = lane >> 5;
  const int wave = uniform((tid >> 6) % NW), kg = uniform((tid >> 6) / NW);  // place among the rows; key group
  const int R = p.q_len * p.group;
  const bool joined = p.chunks > p.batch;
  const Place pl = place(p, 32 * NW);
  const int b = pl.b, kh = pl.kh, chunk = pl.chunk, tile = pl.tile;
  const Chunks ck = pl.ck;
  if (b < 0) return;
  if (joined && tile == 0 && kh == 0) note_chunks(p, b, chunk, ck);
  const int len = uniform(batch_len(p, b));
  const int row0 = tile * 32 * NW + wave * 32, row = row0 + col;
  const int lim = seen_keys(p, len, row);
  const int lim_lo = uniform(seen_keys(p, len, min(row0, R - 1)));  // (rows see more keys further down)
  const int lim_hi = uniform(row0 < R ? seen_keys(p, len, min(row0 + 32, R) - 1) : 0);
  const int kend = uniform(seen_keys(p, len, min((tile + 1) * 32 * NW, R) - 1));
  const int t0 = (chunk - ck.first) * ck.size;
  const int t_end = min(t0 + ck.size, (kend + kTileKeys - 1) / kTileKeys);

  uint4 qf[QS];
  const int i = row / p.group, g = row - i * p.group;
  {
    const char* qp = (const char*)p.q + ((b * (int64_t)p.q_len + i) * p.ldq + (kh * p.group + g) * p.D) * 2;
#pragma unroll
    for (int st = 0; st < QS; ++st) {
      const int c = 2 * st + h;
      qf[st] = row < R && c * 8 < p.D ? *(const uint4*)(qp + c * 16) : make_uint4(0u, 0u, 0u, 0u);
    }
  }

  const int64_t sk = p.ldk * 2, sv = p.ldv * 2;
  const char* kb = (const char*)p.k + (int64_t)b * p.k_len * sk + kh * p.D * 2;
  const char* vb = (const char*)p.v + (int64_t)b * p.k_len * sv + kh * p.D * 2;
  uint32_t ko[NI], vo[NI];
#pragma unroll
  for (int n = 0; n < NI; ++n) {
    const int at = (n * NW + wave) * 64 + lane, r = at / CPR, x = at % CPR;
    const int ck = x ^ k_key<CPR>(r), cv = x ^ v_key<CPR>(r);
    ko[n] = ck * 8 < p.D ? (uint32_t)(r * (int)sk + ck * 16) : kOOB;
    vo[n] = cv * 8 < p.D ? (uint32_t)(r * (int)sv + cv * 16) : kOOB;
  }
  // Fills of successive tiles, the base moving along (few scalar instructions: they are not hidden); rows past
  // the length (and tiles past the end) read as zeros, whatever stands there
  char* const kt = lds + kg * 4 * TILE;  // two tiles of keys
  char* const vt = kt + 2 * TILE;        // and of values
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(kt)) + wave * 1024;
  auto fill = [&](const char*& base, int64_t stride, int& left, const uint32_t* off, uint32_t at) {
    const int valid = min(kTileKeys, left);
    const i32x4 r4 = buffer_rsrc(base, valid > 0 ? (valid - 1) * (int)stride + p.D * 2 : 0);
#pragma unroll
    for (int n = 0; n < NI; ++n) lds_fill16(r4, at + n * NW * 1024, off[n]);
    base += KS * kTileKeys * stride;
    left -= KS * kTileKeys;
  };
  const int first = t0 + kg;  // this group's tiles: first, first + KS, ...
  const char *kp = kb + (int64_t)first * kTileKeys * sk, *vp = vb + (int64_t)first * kTileKeys * sv;
  const int rest = t_end > first ? min(len, t_end * kTileKeys) - first * kTileKeys : 0;  // keys from there on
  int k_left = rest, v_left = rest;
  auto fill_k = [&](auto par_tag) { fill(kp, sk, k_left, ko, lds0 + decltype(par_tag)::value * TILE); };
  auto fill_v = [&](auto par_tag) { fill(vp, sv, v_left, vo, lds0 + (2 + decltype(par_tag)::value) * TILE); };

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = f32x16{};
  float m = -INFINITY, l = 0.0f;
  const float c2 = p.scale * 1.44269504088896340736f;
  const int t_wave = min(t_end, (lim_hi + kTileKeys - 1) / kTileKeys);  // tiles that this wave's rows see
  const int masked = p.causal && p.q_len > 1 ? lim_lo / kTileKeys : INT_MAX;  // the first that some rows see a part of
  int stop = t_wave;                                                          // the tiles from there on are left to add_keys

  // LDS offsets of this lane's operands in a tile: its key row at chunk h, whose other chunks are an XOR
  // away (chunk 2 st + h at st << 5); and its part of V^T for 32-column block d, key group j
  const uint32_t ka = col * RB + ((h ^ k_key<CPR>(col)) << 4);
  uint32_t va[DB][2];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = 8 * j + 4 * h + ((lane & 15) >> 2);
      const int c = d * 4 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      va[d][j] = r * RB + ((c ^ v_key<CPR>(r)) << 4) + (lane & 1) * 8;
    }
  struct KFrag {
    uint4 a[KB];
  };
  struct VFrag {
    uint2 a[DB][2];
  };
  auto read_k = [&](auto par_tag, auto st_tag) {
    constexpr int par = decltype(par_tag)::value, st = decltype(st_tag)::value;
    KFrag f;
#pragma unroll
    for (int n = 0; n < KB; ++n) f.a[n] = *(const uint4*)(kt + (ka ^ (st << 5)) + par * TILE + n * 32 * RB);
    return f;
  };
  auto read_v = [&](auto par_tag, auto ks_tag) {
    constexpr int par = decltype(par_tag)::value, ks = decltype(ks_tag)::value;
    VFrag f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        f.a[d][j] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                  (lds_s16x4)(vt + va[d][j] + par * TILE + ks * 16 * RB)));
    return f;
  };
  auto mul_k = [&](const KFrag& f, auto st_tag, f32x16* s) {
    constexpr int st = decltype(st_tag)::value;
#pragma unroll
    for (int n = 0; n < KB; ++n)
      s[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(f.a[n]), as_bf16x8(qf[st]), s[n], 0, 0, 0);
  };
  auto mul_v = [&](const VFrag& f, uint4 w) {
#pragma unroll
    for (int d = 0; d < DB; ++d)
      o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          as_bf16x8(make_uint4(f.a[d][0].x, f.a[d][0].y, f.a[d][1].x, f.a[d][1].y)), as_bf16x8(w), o[d], 0, 0, 0);
  };

  // Tile t, in the LDS places of its parity: its scores s are there.  While the matrix cores form the next
  // tile's, the vector ALU turns these into weights, a slice per step; operands are read two steps ahead.
  // Then the values are weighted.  (Past the last tile the next scores are of whatever the place holds, and
  // not used.)
  auto step = [&](int t, auto par_tag, f32x16* s, f32x16* next) {
    constexpr std::integral_constant<int, 1 - decltype(par_tag)::value> other{};
    constexpr std::integral_constant<int, 0> c0{};
    constexpr std::integral_constant<int, 1> c1{};
    KFrag kf[3];
    kf[0] = read_k(other, c0);
    kf[1] = read_k(other, c1);
    const int k0 = t * kTileKeys;
    if (k0 + kTileKeys > lim_lo) {
#pragma unroll
      for (int n = 0; n < KB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (k0 + n * 32 + 8 * (e >> 2) + 4 * h + (e & 3) >= lim) s[n][e] = -INFINITY;
    }
    float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < KB; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) tops[e & 3] = fmaxf(tops[e & 3], s[n][e]);
    const float top = half_max(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]))) * c2;
    if (__any(top > m + kSlack)) {  // (m = -inf before the first seen key)
      const float mn = fmaxf(m, top);
      const float keep = exp2_(m - (mn == -INFINITY ? 0.0f : mn));
      m = mn;
      l *= keep;
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] *= keep;
    }
    const float use = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int n = 0; n < KB; ++n) next[n] = f32x16{};
    float sums[2] = {0.0f, 0.0f};
    uint4 pf[2 * KB];
    VFrag vf[2];
    static_for<0, QS>([&](auto st) {
      constexpr int i = decltype(st)::value;
      constexpr int from = 16 * KB * i / QS, to = 16 * KB * (i + 1) / QS;  // weights of a slice
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (i + 2 < QS) kf[(i + 2) % 3] = read_k(other, std::integral_constant<int, i + 2>{});
      if constexpr (i == QS - 1) vf[0] = read_v(par_tag, c0);
      mul_k(kf[i % 3], st, next);
#pragma unroll
      for (int e = from; e < to; ++e) {
        const float w = exp2_(__builtin_fmaf(s[e >> 4][e & 15], c2, -use));
        s[e >> 4][e & 15] = w;
        sums[e & 1] += w;
      }
#pragma unroll
      for (int ks = from / 8; ks < to / 8; ++ks) pf[ks] = pack_weights(s[ks >> 1], ks & 1);
    });
    l += sums[0] + sums[1];
    static_for<0, 2 * KB>([&](auto ks) {
      constexpr int i = decltype(ks)::value;
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (i + 1 < 2 * KB) vf[(i + 1) & 1] = read_v(par_tag, std::integral_constant<int, i + 1>{});
      mul_v(vf[i & 1], pf[i]);
    });
    __builtin_amdgcn_sched_barrier(0);
  };

  auto check = [&](int t, auto par_tag) {
    if (t >= masked && t < stop && holds_not_finite<true, TILE>(vt + decltype(par_tag)::value * TILE)) stop = t;
  };
  // Before step t: its values and the keys of t + 1 have landed for every wave, and every wave is done with
  // the tiles before, whose places keys t + 2 (that of t) and values t + 1 take.
  auto turn = [&](auto same, auto other) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    fill_k(same);
    fill_v(other);
  };
  constexpr std::integral_constant<int, 0> even{};
  constexpr std::integral_constant<int, 1> odd{};
  f32x16 sa[KB], sb[KB];
  fill_k(even);
  asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  fill_k(odd);
  fill_v(even);
#pragma unroll
  for (int n = 0; n < KB; ++n) sa[n] = f32x16{};
  static_for<0, QS>([&](auto st) { mul_k(read_k(even, st), st, sa); });
  for (int t = t0; t < t_end; t += 2 * KS) {
    turn(even, odd);
    check(t + kg, even);
    if (t + kg < stop) step(t + kg, even, sa, sb);
    if (t + KS >= t_end) break;
    turn(odd, even);
    check(t + KS + kg, odd);
    if (t + KS + kg < stop) step(t + KS + kg, odd, sb, sa);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  for (; stop < t_wave; stop += KS)
    add_keys<bf16_t, DB, QS>(p, kb, vb, sk, sv, lim, stop * kTileKeys, (stop + 1) * kTileKeys, qf, c2, o, m, l);
  l = half_sum(l);
  if constexpr (KS > 1) {
    // the second key group hands its results over, lane by lane, in the place of the tiles
    static_assert(KS == 2 && NW * 64 * (16 * DB + 2) * 4 <= (int)sizeof(lds), "the results' place");
    float* const ex = (float*)lds + wave * 64 * (16 * DB + 2) + lane;
    __syncthreads();
    if (kg == 1) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) ex[(d * 16 + e) * 64] = o[d][e];
      ex[16 * DB * 64] = m;
      ex[(16 * DB + 1) * 64] = l;
    }
    __syncthreads();
    if (kg == 1) return;
    const float m1 = ex[16 * DB * 64], l1 = ex[(16 * DB + 1) * 64];
    const float top = fmaxf(m, m1), use = top == -INFINITY ? 0.0f : top;
    const float f0 = exp2_(m - use), f1 = exp2_(m1 - use);
    m = top;
    l = l * f0 + l1 * f1;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = o[d][e] * f0 + ex[(d * 16 + e) * 64] * f1;
  }
  if (row >= R) return;
  if (joined) {
    float* const sums = part_sums(p, kh, row, chunk);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = d * 32 + 8 * e + 4 * h;
        if (c < p.D) *(float4*)(sums + c) = make_float4(o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]);
      }
    if (h == 0) {
      float* out = part_scale(p, kh, row, chunk);
      out[0] = m;
      out[1] = l;
    }
    return;
  }
  // (a row without keys is zero; one whose seen scores are all -inf divides zero by zero, as the softmax does)
  const float inv = 1.0f / l;
  bf16_t* y = (bf16_t*)p.y + (b * (int64_t)p.q_len + i) * p.ldy + (kh * p.group + g) * p.D;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      // columns 8 e + 4 h .. + 3 and 8 (e + 1) + 4 h .. + 3 of this lane become 8 (e + h) .. + 7
      uint32_t w[2][2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int at = 4 * (e + k) + 2 * j;
          w[k][j] = lim > 0 ? pack2_bf16(o[d][at] * inv, o[d][at + 1] * inv) : 0u;
        }
      const u32x2 lo = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
      const u32x2 hi = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
      const int c = d * 32 + 8 * (e + h);
      if (c < p.D) *(uint4*)(y + c) = make_uint4(lo[0], hi[0], lo[1], hi[1]);
    }
}

// Many rows, fp32: four waves of 32 packed rows each share tiles of 32 keys and values, double-buffered in
// LDS, a tile's loads running while the one before is multiplied; bound by the fp32 matrix cores (4096 cycles a
// tile of 64 columns, beside which the softmax is short).  The key axes are not split: choose_attention
// comes here where there are rows enough (16 x 300 over 200, 12 of 128: 105 us, 56 TFLOP/s).
template <int DP, int DC>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void attention_tiles_f32_kernel(AttnParams p) {
  constexpr int NW = 4;
  constexpr int RB = DP * 4, CPR = RB / 16;
  constexpr int TILE = kKeys * RB;
  constexpr int NI = TILE / (NW * 1024);  // loads of a tile per lane
  constexpr int DB = DC / 32, QS = DC / 8;
  __shared__ __align__(1024) char lds[4 * TILE];  // keys, values, keys, values
  static_assert(sizeof(lds) <= kLdsLimit, "LDS");

  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, h = lane >> 5;
  const int wave = uniform(tid >> 6);
  const int R = p.q_len * p.group;
  const Place pl = place(p, 32 * NW);
  const int b = pl.b, kh = pl.kh, tile = pl.tile;
  const int len = uniform(batch_len(p, b));
  const int row0 = tile * 32 * NW + wave * 32, row = row0 + col;
  const int lim = seen_keys(p, len, row);
  const int lim_lo = uniform(seen_keys(p, len, min(row0, R - 1)));  // (rows see more keys further down)
  const int lim_hi = uniform(row0 < R ? seen_keys(p, len, min(row0 + 32, R) - 1) : 0);
  const int kend = uniform(seen_keys(p, len, min((tile + 1) * 32 * NW, R) - 1));
  const int t_end = (kend + kKeys - 1) / kKeys;
  const int t_wave = min(t_end, (lim_hi + kKeys - 1) / kKeys);  // tiles that this wave's rows see

  uint4 qf[QS];
  const int i = row / p.group, g = row - i * p.group;
  {
    const char* qp = (const char*)p.q + ((b * (int64_t)p.q_len + i) * p.ldq + (kh * p.group + g) * p.D) * 4;
#pragma unroll
    for (int st = 0; st < QS; ++st) {
      const int c = 2 * st + h;
      qf[st] = row < R && c * 4 < p.D ? *(const uint4*)(qp + c * 16) : make_uint4(0u, 0u, 0u, 0u);
    }
  }
  const int64_t sk = p.ldk * 4, sv = p.ldv * 4;
  const char* kb = (const char*)p.k + (int64_t)b * p.k_len * sk + kh * p.D * 4;
  const char* vb = (const char*)p.v + (int64_t)b * p.k_len * sv + kh * p.D * 4;
  const uint32_t lds0 = uniform(lds_addr(lds)) + wave * 1024;
  // a tile of keys and values; rows past the length (and tiles past the end) read as zeros, whatever stands there
  auto fill = [&](int par, int t) {
    const int64_t k0 = (int64_t)t * kKeys;
    const int n = t < t_end ? min(kKeys, len - t * kKeys) : 0;
    const i32x4 rk = buffer_rsrc(kb + k0 * sk, n > 0 ? (n - 1) * (int)sk + p.D * 4 : 0);
    const i32x4 rv = buffer_rsrc(vb + k0 * sv, n > 0 ? (n - 1) * (int)sv + p.D * 4 : 0);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int at = (j * NW + wave) * 64 + lane, r = at / CPR, x = at % CPR;
      const int ck = x ^ k_key<CPR>(r), cv = x ^ v_key<CPR>(r);
      lds_fill16(rk, lds0 + par * 2 * TILE + j * NW * 1024, ck * 4 < p.D ? (uint32_t)(r * (int)sk + ck * 16) : kOOB);
      lds_fill16(rv, lds0 + (par * 2 + 1) * TILE + j * NW * 1024, cv * 4 < p.D ? (uint32_t)(r * (int)sv + cv * 16) : kOOB);
    }
  };

  // LDS offsets of this lane's operands in a tile: its key row at chunk h, whose other chunks are an XOR away; and
  // column col of value rows 4 h and on (v_key(r + 4 h) = v_key(r) ^ h)
  static_assert(CPR >= 16, "swizzle keys of 4 bits");
  const uint32_t ka = col * RB + ((h ^ k_key<CPR>(col)) << 4);
  const uint32_t va = 4 * h * RB + (((col >> 2) ^ h) << 4) + (col & 3) * 4;

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = f32x16{};
  float m = -INFINITY, l = 0.0f;
  const float c2 = p.scale * 1.44269504088896340736f;
  const int masked = p.causal && p.q_len > 1 ? lim_lo / kKeys : INT_MAX;  // the first tile that some rows see a part of
  int stop = t_wave;                                                      // the tiles from there on are left to add_keys
  auto compute = [&](int par, int t) {
    const char* kt = lds + par * 2 * TILE;
    const char* vt = kt + TILE;
    f32x16 s{};
#pragma unroll
    for (int st = 0; st < QS; ++st) {
      const f32x4 a = *(const f32x4*)(kt + (ka ^ (st % 8 << 5)) + st / 8 * 256);
      const f32x4 q = __builtin_bit_cast(f32x4, qf[st]);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], q[e], s, 0, 0, 0);
    }
    const int k0 = t * kKeys + 4 * h;
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = k0 + 8 * (e >> 2) + (e & 3) < lim ? s[e] * c2 : -INFINITY;
      top = fmaxf(top, s[e]);
    }
    const float mn = fmaxf(m, half_max(top));
    const float use = mn == -INFINITY ? 0.0f : mn;  // (no key seen yet: every weight is zero)
    const float keep = exp2_(m - use);
    m = mn;
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = exp2_(s[e] - use);
      sum += s[e];
    }
    l = l * keep + sum;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] *= keep;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = 8 * (e >> 2) + (e & 3);  // (and 4 h)
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const float vf = *(const float*)(vt + (va ^ ((v_key<CPR>(r) & 7) << 4)) + r * RB + ((d ^ (v_key<CPR>(r) >> 3)) * 128));
        o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[e], o[d], 0, 0, 0);
      }
    }
  };

  fill(0, 0);
  for (int t = 0, par = 0; t < t_end; ++t, par ^= 1) {
    // tile t has landed for every wave, and every wave is done with the one before, whose place t + 1 takes
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    fill(par ^ 1, t + 1);
    if (t >= masked && t < stop && holds_not_finite<false, TILE>(lds + (par * 2 + 1) * TILE)) stop = t;
    if (t < stop) compute(par, t);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  for (; stop < t_wave; ++stop)
    add_keys<float, DB, QS>(p, kb, vb, sk, sv, lim, stop * kKeys, (stop + 1) * kKeys, qf, c2, o, m, l);
  l = half_sum(l);
  if (row >= R) return;
  // (a row without keys is zero; one whose seen scores are all -inf divides zero by zero, as the softmax does)
  float* const y = (float*)p.y + (b * (int64_t)p.q_len + i) * p.ldy + (kh * p.group + g) * p.D;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = d * 32 + 8 * e + 4 * h;
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = lim > 0 ? o[d][4 * e + j] / l : 0.0f;
      if (c < p.D) *(float4*)(y + c) = make_float4(v[0], v[1], v[2], v[3]);
    }
}

// Joins the chunks of a packed row: D / 4 lanes (of 64 / 32 / 16), 4 columns each, and `split` such groups a
// row that take the chunks in turn, so that many chunks are on their way together where there are few rows
// (one token over 32768 keys, 16 heads on one of 128, 16 rows of 85 chunks: 39 us by one group, 17 by eight).
__global__ __launch_bounds__(256) void attention_join_kernel(AttnParams p, int lanes, int split) {
  __shared__ float4 part[256];
  __shared__ float2 part_ml[256];
  const int R = p.q_len * p.group;
  // rows of one sequence per workgroup row (blockIdx.y), so that a wave has one set of chunks
  const int b = blockIdx.y;
  const int len = batch_len(p, b);
  const int2 ck = len > 0 ? ((const int2*)p.ws)[b] : make_int2(0, 0);  // first chunk, count
  const int slot = threadIdx.x / lanes, g0 = slot % split;
  const int at = blockIdx.x * (256 / lanes / split) + slot / split;  // (key head, packed row)
  const int c = threadIdx.x % lanes * 4;
  const bool live = at < p.kv_heads * R && c < p.D;
  const int kh = live ? at / R : 0, row = live ? at - kh * R : 0;
  // eight chunks at a time, their loads on the way together
  float top = -INFINITY, total = 0.0f;
  float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (live) {
    const float* ml = part_scale(p, kh, row, ck.x);
    const float* os = part_sums(p, kh, row, ck.x) + c;
    for (int s0 = g0; s0 < ck.y; s0 += 8 * split) {
      float2 m[8];
      float4 x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int s = min(s0 + k * split, ck.y - 1);
        m[k] = *(const float2*)(ml + 2 * s);
        x[k] = *(const float4*)(os + (int64_t)s * p.D);
      }
      float most = top;
#pragma unroll
      for (int k = 0; k < 8; ++k) most = fmaxf(most, m[k].x);
      const float use = most == -INFINITY ? 0.0f : most;
      const float keep = exp2_(top - use);
      top = most;
      total *= keep;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] *= keep;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (s0 + k * split >= ck.y) break;
        const float f = exp2_(m[k].x - use);
        total += m[k].y * f;
        v[0] += x[k].x * f, v[1] += x[k].y * f, v[2] += x[k].z * f, v[3] += x[k].w * f;
      }
    }
  }
  if (split > 1) {  // (the groups in order, so that a sum does not depend on their timing)
    part[threadIdx.x] = make_float4(v[0], v[1], v[2], v[3]);
    part_ml[threadIdx.x] = make_float2(top, total);
    __syncthreads();
    if (g0 > 0) return;
    float most = top;
    for (int k = 1; k < split; ++k) most = fmaxf(most, part_ml[threadIdx.x + k * lanes].x);
    const float use = most == -INFINITY ? 0.0f : most;
    const float keep = exp2_(top - use);
    total *= keep;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] *= keep;
    for (int k = 1; k < split; ++k) {
      const float2 m = part_ml[threadIdx.x + k * lanes];
      const float4 x = part[threadIdx.x + k * lanes];
      const float f = exp2_(m.x - use);
      total += m.y * f;
      v[0] += x.x * f, v[1] += x.y * f, v[2] += x.z * f, v[3] += x.w * f;
    }
  }
  if (!live) return;
  const bool any = seen_keys(p, len, row) > 0;
  const int i = row / p.group, g = row - i * p.group;
  const int64_t out = (b * (int64_t)p.q_len + i) * p.ldy + (kh * p.group + g) * p.D + c;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = any ? v[j] / total : 0.0f;
  if (p.f32)
    *(float4*)((float*)p.y + out) = make_float4(v[0], v[1], v[2], v[3]);
  else
    *(uint2*)((bf16_t*)p.y + out) = make_uint2(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]));
}

// waves of a workgroup of the rows kernel: as many as the LDS has tiles for
int row_waves(const AttnParams& p) { return p.D > 128 ? 2 : p.D > 64 || p.f32 ? 4 : 8; }

// workgroups along the rows
int row_blocks(const AttnParams& p) {
  return ceil_div((int64_t)p.q_len * p.group, p.tile_rows);
}

}  // namespace

// Chunks of each sequence for the tiles kernel on `blocks` workgroups a chunk: the number of least modelled time (us), of
// the tiles of 64 keys that a workgroup takes one after another, slower where two share a CU, and of the results' way
// through memory to the join.  Measured, whole and in the chunks of this rule: 1 x 1024 over 1024, 12 heads of 64, 11.4 as
// both (18.8 in two chunks); 1 x 1024 over 4096, 8 of 128, 68 and 38; 4 x 40 over 8192, 8 of 64, 54 and 20.
int split_tiles(const AttnParams& p, int64_t blocks) {
  const double tile = p.D <= 64 ? 0.4 : p.D <= 96 ? 0.93 : p.D <= 128 ? 1.03 : p.D <= 192 ? 2.1 : 2.65;
  const double shared = p.D <= 64 ? 1.0 : 0.4;  // (at 64 columns, which the vector ALU bounds, a second workgroup gains nothing)
  const double tiles = ceil_div(p.k_len, kTileKeys);
  const double part = 8e-6 / 4.1 * p.D * p.batch * p.kv_heads * p.q_len * p.group;  // a chunk's sums, written and read
  int best = 1;
  double least = INFINITY;
  const int64_t most = std::min<int64_t>((p.D > 128 ? 256 : 512) / blocks, ceil_div(p.k_len, 4 * kTileKeys));
  for (int n = 1; n <= most; ++n) {
    const double t = tiles / n * tile * (1.0 + shared * std::max(0.0, blocks * n / 256.0 - 1.0)) + (n > 1 ? 6.0 + part * n : 0.0);
    if (t < least) least = t, best = n;
  }
  return best;
}

// The kernel and the split.  bf16: the shared tiles take more than 32 packed rows (with fewer three of
// their four waves would idle).  fp32 products are bound by the matrix cores either way: the shared
// tiles where their workgroups of 128 rows fill the chip, or where the keys are too few for the
// waves of the rows kernel (us, tiles and rows kernel: 16 x 600 over 60 keys, 16 heads on one of 128,
// 72, 218; 16 x 300 over 200, 12 of 128, 106, 134; 16 x 100 over 100, 12 of 64, 16, 20; but 8 x 512 over
// 512, 12 of 64, 84, 77; 4 x 512 over 256, 8 of 128, 45, 36).
void choose_attention(AttnParams& p) {
  const int64_t rows = p.q_len * (int64_t)p.group;
  const int64_t quads = (int64_t)p.batch * p.kv_heads * ceil_div(rows, 128);
  const bool tiled = rows > 32 && (!p.f32 || quads >= (p.D <= 64 ? 512 : 256) || (p.k_len <= 4 * kKeys && quads >= 128));
  // Up to 64 columns a head, two waves along the rows and two along the keys where 128-row workgroups would
  // not fill the chip twice: causal 1 x 2048, 16 heads of 64: 30.5 us as 256 workgroups of 128 rows, 21.4 as
  // 512 of 64; 128 columns need the LDS of a CU for that and lose (1 x 1024, 32 over 8 of 128: 25.1, 29.1).
  const bool halves = tiled && !p.f32 && p.D <= 64 && quads <= 320;
  p.tile_rows = tiled ? (halves ? 64 : 128) : kCols;
  p.tile_keys = tiled && !p.f32 ? kTileKeys : kKeys;
  const int64_t blocks = (int64_t)p.batch * p.kv_heads * row_blocks(p);
  int64_t chunks = p.batch;
  if (!tiled) {
    // Rows: one workgroup has a CU to itself; three rounds of its waves in each at least, which take as
    // long as the join
    chunks = std::min<int64_t>(256 / std::max<int64_t>(1, blocks / p.batch),
                               p.batch * (ceil_div(p.k_len, kKeys * row_waves(p)) / 3));
  } else if (blocks < 256) {
    chunks = p.batch * split_tiles(p, blocks);
  }
  p.chunks = chunks < 2 * (int64_t)p.batch ? p.batch : (int)(p.batch > 64 ? chunks / p.batch * p.batch : chunks);
}

const char* attention_name(const AttnParams& p) {
  if (p.tile_rows > kCols) return p.f32 ? "attention_tiles_f32" : "attention_tiles";
  return p.f32 ? "attention_rows_f32" : "attention_rows";
}

int64_t attn_workspace(const AttnParams& p) {
  if (p.chunks <= p.batch) return 0;
  return (head_floats(p) + (int64_t)p.kv_heads * p.q_len * p.group * p.chunks * (p.D + 2)) * 4;
}

hipError_t launch_attention(const AttnParams& p, hipStream_t s) {
  if (p.D < 8 || p.D > 256 || p.D % 8 != 0 || p.chunks < p.batch) return hipErrorInvalidValue;
  const int grid = p.chunks * p.kv_heads * row_blocks(p);
  if (p.tile_rows > kCols) {
    if (p.f32) {
      if (p.D <= 32) attention_tiles_f32_kernel<64, 32><<<grid, 256, 0, s>>>(p);
      else if (p.D <= 64) attention_tiles_f32_kernel<64, 64><<<grid, 256, 0, s>>>(p);
      else if (p.D <= 96) attention_tiles_f32_kernel<128, 96><<<grid, 256, 0, s>>>(p);
      else if (p.D <= 128) attention_tiles_f32_kernel<128, 128><<<grid, 256, 0, s>>>(p);
      else if (p.D <= 192) attention_tiles_f32_kernel<256, 192><<<grid, 256, 0, s>>>(p);
      else attention_tiles_f32_kernel<256, 256><<<grid, 256, 0, s>>>(p);
    } else if (p.tile_rows == 64) {
      if (p.D <= 32) attention_tiles_kernel<64, 32, 2><<<grid, 256, 0, s>>>(p);
      else attention_tiles_kernel<64, 64, 2><<<grid, 256, 0, s>>>(p);
    } else {
      if (p.D <= 32) attention_tiles_kernel<64, 32, 1><<<grid, 256, 0, s>>>(p);
      else if (p.D <= 64) attention_tiles_kernel<64, 64, 1><<<grid, 256, 0, s>>>(p);
      else if (p.D <= 96) attention_tiles_kernel<128, 96, 1><<<grid, 256, 0, s>>>(p);
      else if (p.D <= 128) attention_tiles_kernel<128, 128, 1><<<grid, 256, 0, s>>>(p);
      else if (p.D <= 192) attention_tiles_kernel<256, 192, 1><<<grid, 256, 0, s>>>(p);
      else attention_tiles_kernel<256, 256, 1><<<grid, 256, 0, s>>>(p);
    }
    return hipGetLastError();
  }
  if (p.f32) {
    if (p.D <= 32) attention_rows_kernel<float, 64, 32, 4><<<grid, 256, 0, s>>>(p);
    else if (p.D <= 64) attention_rows_kernel<float, 64, 64, 4><<<grid, 256, 0, s>>>(p);
    else if (p.D <= 96) attention_rows_kernel<float, 128, 96, 4><<<grid, 256, 0, s>>>(p);
    else if (p.D <= 128) attention_rows_kernel<float, 128, 128, 4><<<grid, 256, 0, s>>>(p);
    else if (p.D <= 192) attention_rows_kernel<float, 256, 192, 2><<<grid, 128, 0, s>>>(p);
    else attention_rows_kernel<float, 256, 256, 2><<<grid, 128, 0, s>>>(p);
  } else {
    if (p.D <= 64) attention_rows_kernel<bf16_t, 64, 64, 8><<<grid, 512, 0, s>>>(p);
    else if (p.D <= 128) attention_rows_kernel<bf16_t, 128, 128, 4><<<grid, 256, 0, s>>>(p);
    else attention_rows_kernel<bf16_t, 256, 256, 2><<<grid, 128, 0, s>>>(p);
  }
  return hipGetLastError();
}

hipError_t launch_attention_join(const AttnParams& p, hipStream_t s) {
  const int lanes = p.D <= 64 ? 16 : p.D <= 128 ? 32 : 64;
  const int64_t rows = (int64_t)p.kv_heads * p.q_len * p.group;
  int split = 1;
  while (split < 256 / lanes && split * 8 < p.chunks && rows * p.batch * split * lanes < 256 * 256) split *= 2;
  const dim3 grid(ceil_div(rows, 256 / lanes / split), p.batch);
  attention_join_kernel<<<grid, 256, 0, s>>>(p, lanes, split);
  return hipGetLastError();
}

}  // namespace byoc
