// Rules on logits, before a token is chosen from them.  With n_t the occurrences of
// token t among the tokens that a sequence has generated (and among the drafted tokens that
// lead to a row), s_t whether t is among them or in the prompt:
//   x = s_t ? (x > 0 ? x / r : x r) : x
//   x = x - frequency n_t - (n_t > 0 ? presence : 0)
//   x = x + bias_t             (the last of the entries for t)
//   x = -inf where the mask's bit t is 0
// in float32, rounded once.
//
// A workgroup owns some rows of one sequence and takes chunks of the vocabulary in turn.  For each it counts the history's
// tokens, which it holds in registers, in an LDS table of the chunk (integer additions and maxima,
// whose order does not matter) and lists those that it met; each row of the chunk then passes through LDS,
// where the listed tokens' logits are changed in place, while the next one's loads are on their way.
// So the vector ALU, whose 16 lanes a SIMD would bound a pass that tests and divides at every
// token, has 2 to 3 instructions a token to do (256 rows of 131072 bf16 with every rule, 143 MB: 59 us so tested, 45
// here, 3.2 TB/s; a mask alone, which needs no LDS, 27 us, 5.1 TB/s).  What is left above the copy's time is that
// of the two barriers a row, which leave the memory idle for a part of it.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "row_chunk.h"
#include "tree_paths.h"

namespace byoc {
namespace {

constexpr int kStagedValues = 1024;  // bias values that go to LDS

// A table word: the count, `prompt` (met in the prompt), `listed` (a drafted token), and
// the last bias entry for the token, and 1, in the bits above.
struct Word {
  uint32_t prompt, listed;
  int shift;
};
__device__ __forceinline__ Word word_of(const LogitsParams& p) {
  return Word{1u << p.count_bits, 2u << p.count_bits, p.count_bits + 2};
}

// Elements i0 + tid, i0 + tid + NT, ... of a list, K of them.
template <int NT, int K>
struct Ahead {
  int v[K];
  __device__ __forceinline__ void load(const int* a, int i0, int n) {
#pragma unroll
    for (int u = 0; u < K; ++u)
      if (i0 + u * NT < n) v[u] = a[min(i0 + u * NT + (int)threadIdx.x, n - 1)];
  }
  template <class F>
  __device__ __forceinline__ void each(int i0, int n, F visit) const {
#pragma unroll
    for (int u = 0; u < K; ++u) {
      if (i0 + u * NT >= n) break;
      const int i = i0 + u * NT + (int)threadIdx.x;
      if (i < n) visit(i, v[u]);
    }
  }
};

__device__ __forceinline__ void all_done() { __builtin_amdgcn_s_waitcnt(0x0F70); }  // vmcnt(0)

template <bool F32>
__device__ __forceinline__ float value_of(uint32_t bits) {
  return __uint_as_float(F32 ? bits : bits << 16);
}

template <bool F32, int NT, bool RULES, bool MASK>
__global__ __launch_bounds__(NT, NT == 1024 ? 8 : 4) void logits_kernel(LogitsParams p) {
  constexpr int C = NT * 8;  // tokens of a chunk
  constexpr int LIST = C / 2;  // of them are listed; where more were met, all of the chunk is gone through
  typedef typename std::conditional<F32, uint32_t, uint16_t>::type Bits;
  extern __shared__ __align__(16) char lds[];
  uint32_t* const table = (uint32_t*)lds;          // [C], zero between chunks
  Bits* const staged = (Bits*)(lds + C * 4);       // [C]: a row's logits
  uint16_t* const list = (uint16_t*)(staged + C);  // [LIST]: the tokens met
  float* const values = (float*)(list + LIST);     // [kStagedValues] bias values
  uint32_t* const tree = (uint32_t*)(values + (p.bias_tokens ? kStagedValues : 0));  // with drafts: their paths, then their tokens
  __shared__ int listed[2];
  const int tid = threadIdx.x;
  const int chunks = (p.cols_out + C - 1) / C, groups = (p.rows + p.group - 1) / p.group;
  const int parts = (chunks + p.chunks - 1) / p.chunks;
  const int at0 = blockIdx.x / parts, q0 = (blockIdx.x - at0 * parts) * p.chunks, q1 = min(q0 + p.chunks, chunks);
  const int b = at0 / groups, r0 = (at0 - b * groups) * p.group, r1 = min(r0 + p.group, p.rows);

  // the rows of the chunks, one after the other; the next one's loads are always on their way.  (Whole chunks are
  // loaded and stored without a branch and the last one waits for its accesses by itself: the wait for a
  // row's loads is then not one for the stores of the row before, which were given out after them.)
  Chunk<F32> x;
  uint32_t allowed = 0xFFu;
  auto load = [&](int q, int r) {
    const int64_t row = (int64_t)b * p.rows + r;
    const int col = q * C + tid * 8;
    const uint8_t* const m = MASK ? (const uint8_t*)(p.mask + row * ((p.V + 31) / 32)) : nullptr;
    if ((q + 1) * C <= p.V) {
      x.load(p.x, row * p.ldx, col, INT_MAX);
      if constexpr (MASK) allowed = m[col >> 3];
    } else {
      x.load(p.x, row * p.ldx, col, p.V);
      if constexpr (MASK) allowed = col < p.V ? m[col >> 3] : 0u;
      all_done();
    }
  };
  load(q0, r0);

  float rep = 1.0f, pres = 0.0f, freq = 0.0f;
  const Word wd = word_of(p);
  const int* const h = p.history + (int64_t)b * p.T;
  const int* const bt = p.bias_tokens + (int64_t)b * p.E;
  const float* const bv = p.bias_values + (int64_t)b * p.E;
  int len = 0, prompt = 0;
  constexpr int KH = NT == 1024 ? 4 : 8, KB = 1;  // held in registers; longer lists are read again for each chunk
  Ahead<NT, KH> ha;
  Ahead<NT, KB> ba;
  TreePaths paths{};
  int* const tokens = (int*)tree + (p.drafts ? tree_lds_bytes(p.rows) / 4 : 0);
  if constexpr (RULES) {
    if (p.history) {
      ha.load(h, 0, p.T);  // (before the length is known)
      rep = p.strengths[b * 3], pres = p.strengths[b * 3 + 1], freq = p.strengths[b * 3 + 2];
      len = min(max(p.lengths[b], 0), p.T), prompt = p.prompts[b];
    }
    if (p.bias_tokens) {
      ba.load(bt, 0, p.E);
      for (int e = tid; e < min(p.E, kStagedValues); e += NT) values[e] = bv[e];
    }
    for (int i = tid; i < C / 4; i += NT) ((uint4*)table)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (tid < 2) listed[tid] = 0;
    if (p.drafts) {
      const int64_t at = (int64_t)b * p.rows;
      for (int j = tid; j < p.rows; j += NT) tokens[j] = p.drafts[at + j];
      paths = form_paths<NT>(p.parents + at, p.rows, tree);
    }
    lds_barrier();
  }

  for (int q = q0; q < q1; ++q) {
    const int c0 = q * C, end = min(c0 + C, p.V), col = c0 + tid * 8;
    auto mine = [&](int t) { return t >= c0 && t < end; };
    int* const n_listed = &listed[q & 1];
    if constexpr (RULES) {
      auto meet = [&](int t, uint32_t old) {
        if (old != 0u) return;
        const int i = atomicAdd(n_listed, 1);
        if (i < LIST) list[i] = (uint16_t)t;
      };
      if (p.bias_tokens) {
        auto visit = [&](int e, int t) {
          if (mine(t)) meet(t - c0, atomicMax(&table[t - c0], (uint32_t)(e + 1) << wd.shift));
        };
        ba.each(0, p.E, visit);
        for (int e0 = KB * NT; e0 < p.E; e0 += 4 * NT) {
          Ahead<NT, 4> a;
          a.load(bt, e0, p.E);
          a.each(e0, p.E, visit);
        }
        lds_barrier();  // (maxima of whole words before there are counts in them)
      }
      if (p.history) {
        auto visit = [&](int j, int t) {
          if (!mine(t) || j >= len) return;
          uint32_t* const w = &table[t - c0];
          meet(t - c0, j < prompt ? atomicOr(w, wd.prompt) : atomicAdd(w, 1u));
        };
        ha.each(0, p.T, visit);
        for (int j0 = KH * NT; j0 < len; j0 += 4 * NT) {
          Ahead<NT, 4> a;
          a.load(h, j0, p.T);
          a.each(j0, p.T, visit);
        }
      }
      if (p.drafts)
        for (int j = tid; j < p.rows; j += NT)
          if (mine(tokens[j])) meet(tokens[j] - c0, atomicOr(&table[tokens[j] - c0], wd.listed));
    }
    // the drafted tokens that lead to a row, counted while it is at work
    auto count_path = [&](int r, uint32_t by) {
      for (int j = tid; j <= r; j += NT)
        if (paths.word(r, j >> 5) >> (j & 31) & 1u && mine(tokens[j])) atomicAdd(&table[tokens[j] - c0], by);
    };

    for (int r = r0; r < r1; ++r) {
      uint32_t v[F32 ? 8 : 4];
      const uint32_t bits = allowed;
      if constexpr (F32) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __float_as_uint(x.v[k]);
      } else {
        v[0] = x.u.x, v[1] = x.u.y, v[2] = x.u.z, v[3] = x.u.w;
      }
      uint4* const d = (uint4*)(staged + tid * 8);
      if constexpr (RULES) {
#pragma unroll
        for (int k = 0; k < (F32 ? 2 : 1); ++k) d[k] = make_uint4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
      }
      const bool last = r + 1 == r1;
      if (!last) load(q, r + 1);
      else if (q + 1 < q1) load(q + 1, r0);
      if constexpr (RULES) {
        if (p.drafts) {
          if (r > r0) count_path(r - 1, ~0u);
          count_path(r, 1u);
        }
        lds_barrier();
        const int met = *n_listed, n = met > LIST ? C : met;
        for (int i = tid; i < n; i += NT) {
          const int t = met > LIST ? i : list[i];
          const uint32_t w = table[t], made = w & (wd.prompt - 1), e = w >> wd.shift;
          float y = value_of<F32>(staged[t]);
          if (made || (w & wd.prompt)) y = y > 0.0f ? y / rep : y * rep;
          if (made) y = y - freq * (float)made - pres;
          if (e) y += e <= kStagedValues ? values[e - 1] : bv[e - 1];
          staged[t] = (Bits)(F32 ? __float_as_uint(y) : (uint32_t)f32_to_bf16(y));
          if (last) table[t] = 0u;
        }
        if (last && tid == 0) listed[(q + 1) & 1] = 0;
        lds_barrier();
#pragma unroll
        for (int k = 0; k < (F32 ? 2 : 1); ++k) {
          const uint4 c = d[k];
          v[4 * k] = c.x, v[4 * k + 1] = c.y, v[4 * k + 2] = c.z, v[4 * k + 3] = c.w;
        }
      }
      if constexpr (MASK) {
#pragma unroll
        for (int k = 0; k < (F32 ? 8 : 4); ++k) {
          // all bits of a value that stays, none of one that becomes -inf
          const uint32_t lo = (uint32_t)((int)(bits << (31 - (F32 ? k : 2 * k))) >> 31);
          if constexpr (F32) {
            v[k] = (v[k] & lo) | (0xFF800000u & ~lo);
          } else {
            const uint32_t hi = (uint32_t)((int)(bits << (30 - 2 * k)) >> 31);
            const uint32_t keep = (lo & 0xFFFFu) | (hi & 0xFFFF0000u);
            v[k] = (v[k] & keep) | (0xFF80FF80u & ~keep);
          }
        }
      }
      // (the columns past the vocabulary, where the output has some, are zeros)
      Bits* const y = (Bits*)p.y + ((int64_t)b * p.rows + r) * p.ldy + col;
      auto store = [&] {
        if constexpr (F32) {
#pragma unroll
          for (int k = 0; k < 8; k += 4)
            *(F32x4u*)(y + k) = F32x4u{__uint_as_float(v[k]), __uint_as_float(v[k + 1]), __uint_as_float(v[k + 2]), __uint_as_float(v[k + 3])};
        } else {
          *(Bf16x8u*)y = Bf16x8u{v[0], v[1], v[2], v[3]};
        }
      };
      if (c0 + C <= p.V) {
        store();
      } else {
        if (col + 8 <= p.V) {
          store();
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (col + k < p.cols_out) y[k] = (Bits)(col + k >= p.V ? 0u : F32 ? v[k] : v[k >> 1] >> (16 * (k & 1)));
        }
        all_done();
      }
    }
  }
}

template <bool F32, int NT, bool RULES, bool MASK>
hipError_t launch_as(const LogitsParams& p, hipStream_t s) {
  constexpr int C = NT * 8;
  const int bytes = (RULES ? C * (4 + (F32 ? 4 : 2) + 1) : 0) + (p.bias_tokens ? kStagedValues * 4 : 0) +
                    (p.drafts ? tree_lds_bytes(p.rows) + p.rows * 4 : 0);
  const int64_t grid = (int64_t)ceil_div(ceil_div(p.cols_out, C), p.chunks) * ceil_div(p.rows, p.group) * p.batch;
  logits_kernel<F32, NT, RULES, MASK><<<(unsigned)grid, NT, bytes, s>>>(p);
  return hipGetLastError();
}

template <bool F32, int NT>
hipError_t launch_rules(const LogitsParams& p, hipStream_t s) {
  const bool rules = p.history || p.bias_tokens;
  if (rules && p.mask) return launch_as<F32, NT, true, true>(p, s);
  if (rules) return launch_as<F32, NT, true, false>(p, s);
  if (p.mask) return launch_as<F32, NT, false, true>(p, s);
  return hipErrorInvalidValue;
}

}  // namespace

// Threads, rows and chunks of a workgroup.  Large calls and long histories (every chunk looks at all of one) take
// 1024 threads, whose chunks are 8192 tokens: 256 rows of 131072 after 2048 tokens 45 us, 52 with 512; 32 rows
// of 60000 after 16000 13.0 and 17.5; but 2 x 60 rows of 100000 18.7, 17.5 with 512, as fewer rows follow one
// another; 250 rows of 3000 6.8, and 6.2 with 256, whose chunks are 2048.  More rows or chunks than the chip
// holds workgroups for follow one another in them, which starts the next one's loads early and keeps the history
// in registers: 256 rows of 131072, 16 chunks each, 64 us one by one, 45 eight by eight.
void choose_logits(LogitsParams& p) {
  p.count_bits = 0;  // (with the other fields at most 32 bits: parse_graph sees to it)
  while (((int64_t)p.T + kMaxTree) >> p.count_bits) ++p.count_bits;
  const int64_t all = (int64_t)p.batch * p.rows * p.cols_out;
  p.threads = all >= 1 << 24 || p.T > 8192 ? 1024 : p.cols_out > 4096 ? 512 : 256;
  const int64_t blocks = (int64_t)p.batch * ceil_div(p.cols_out, p.threads * 8), room = p.threads == 1024 ? 512 : 768;
  p.group = (int)std::min<int64_t>(p.rows, std::max<int64_t>(1, ceil_div(blocks * p.rows, room)));
  p.chunks = (int)std::max<int64_t>(1, ceil_div(blocks * ceil_div(p.rows, p.group), room));
}

hipError_t launch_logits(const LogitsParams& p, hipStream_t s) {
  if (p.drafts && p.rows > kMaxTree) return hipErrorInvalidValue;
  if (p.threads == 1024) return p.f32 ? launch_rules<true, 1024>(p, s) : launch_rules<false, 1024>(p, s);
  if (p.threads == 512) return p.f32 ? launch_rules<true, 512>(p, s) : launch_rules<false, 512>(p, s);
  return p.f32 ? launch_rules<true, 256>(p, s) : launch_rules<false, 256>(p, s);
}

}  // namespace byoc
