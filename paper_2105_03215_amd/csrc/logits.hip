// Rules on logits, before a token is chosen from them.  With n_t the occurrences of
// token t among the tokens that a sequence has generated (and among the drafted tokens that
// lead to a row), s_t whether t is among them or in the prompt:
//   x = s_t ? (x > 0 ? x / r : x r) : x
//   x = x - frequency n_t - (n_t > 0 ? presence : 0)
//   x = x + bias_t             (the last of the entries for t)
//   x = -inf where the mask's bit t is 0
// in float32, rounded once.
//
// A workgroup owns a chunk of the vocabulary of one sequence: it counts the history's
// tokens of its chunk in an LDS table (integer additions, whose order does not matter) and
// then streams its rows' logits past it.
#include <algorithm>

#include "row_chunk.h"
#include "tree_paths.h"

namespace byoc {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kPrompt = 0x80000000u;  // of a table word: seen in the prompt; the bits below count

template <bool F32, int IT, bool PEN, bool BIAS, bool MASK>
__global__ __launch_bounds__(kThreads) void logits_kernel(LogitsParams p) {
  constexpr int C = kThreads * 8 * IT;  // tokens of a chunk
  extern __shared__ __align__(16) uint32_t lds[];
  uint32_t* const table = lds;                          // [C] with PEN
  uint32_t* const entry = lds + (PEN ? C : 0);          // [C] with BIAS: the last entry for a token, and 1
  uint32_t* const tree = entry + (BIAS ? C : 0);        // with drafts: their paths, then their tokens
  const int tid = threadIdx.x;
  const int chunks = (p.cols_out + C - 1) / C, groups = (p.rows + p.group - 1) / p.group;
  const int at0 = blockIdx.x / chunks, c0 = (blockIdx.x - at0 * chunks) * C;
  const int b = at0 / groups, r0 = (at0 - b * groups) * p.group, r1 = min(r0 + p.group, p.rows);
  const int end = min(c0 + C, p.V);

  Chunk<F32> x[IT];
  auto load = [&](int r) {
#pragma unroll
    for (int i = 0; i < IT; ++i) x[i].load(p.x, ((int64_t)b * p.rows + r) * p.ldx, c0 + (i * kThreads + tid) * 8, p.V);
  };
  load(r0);

  float rep = 1.0f, pres = 0.0f, freq = 0.0f;
  TreePaths paths{};
  int* tokens = nullptr;
  if constexpr (PEN || BIAS) {
    for (int i = tid; i < (PEN + BIAS) * C / 4; i += kThreads) ((uint4*)lds)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
  }
  if constexpr (PEN) {
    rep = p.strengths[b * 3], pres = p.strengths[b * 3 + 1], freq = p.strengths[b * 3 + 2];
    const int len = min(max(p.lengths[b], 0), p.T), prompt = p.prompts[b];
    const int* h = p.history + (int64_t)b * p.T;
    for (int j = tid; j < len; j += kThreads) {
      const int t = h[j];
      if (t < c0 || t >= end) continue;
      if (j < prompt) atomicOr(&table[t - c0], kPrompt);
      else atomicAdd(&table[t - c0], 1u);
    }
    if (p.drafts) {
      const int64_t at = (int64_t)b * p.rows;
      tokens = (int*)tree + tree_lds_bytes(p.rows) / 4;
      for (int j = tid; j < p.rows; j += kThreads) tokens[j] = p.drafts[at + j];
      paths = form_paths<kThreads>(p.parents + at, p.rows, tree);
    }
  }
  if constexpr (BIAS) {
    const int* bt = p.bias_tokens + (int64_t)b * p.E;
    for (int e = tid; e < p.E; e += kThreads) {
      const int t = bt[e];
      if (t >= c0 && t < end) atomicMax(&entry[t - c0], (uint32_t)e + 1u);
    }
  }

  for (int r = r0; r < r1; ++r) {
    if (r > r0) load(r);
    // the drafted tokens that lead to the row, counted for it alone
    auto count_path = [&](uint32_t by) {
      for (int j = tid; j <= r; j += kThreads) {
        const int t = tokens[j];
        if (paths.word(r, j >> 5) >> (j & 31) & 1u && t >= c0 && t < end) atomicAdd(&table[t - c0], by);
      }
    };
    if (PEN && p.drafts) count_path(1u);
    if constexpr (PEN || BIAS) __syncthreads();
    const int64_t row = (int64_t)b * p.rows + r;
    const uint8_t* mask = MASK ? (const uint8_t*)(p.mask + row * ((p.V + 31) / 32)) : nullptr;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int at = (i * kThreads + tid) * 8, col = c0 + at;
      if (col >= p.cols_out) break;
      float v[8];
      x[i].get(v);
      if constexpr (PEN) {
        const uint4 n0 = *(const uint4*)(table + at), n1 = *(const uint4*)(table + at + 4);
        const uint32_t n[8] = {n0.x, n0.y, n0.z, n0.w, n1.x, n1.y, n1.z, n1.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (n[e] == 0u) continue;
          v[e] = v[e] > 0.0f ? v[e] / rep : v[e] * rep;
          const uint32_t made = n[e] & ~kPrompt;
          if (made) v[e] = v[e] - freq * (float)made - pres;
        }
      }
      if constexpr (BIAS) {
        const uint4 n0 = *(const uint4*)(entry + at), n1 = *(const uint4*)(entry + at + 4);
        const uint32_t n[8] = {n0.x, n0.y, n0.z, n0.w, n1.x, n1.y, n1.z, n1.w};
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (n[e]) v[e] += p.bias_values[(int64_t)b * p.E + n[e] - 1];
      }
      if constexpr (MASK) {
        const uint32_t bits = col < p.V ? mask[col >> 3] : 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!(bits >> e & 1u)) v[e] = -INFINITY;
      }
      if (col + 8 > p.V) {  // (the columns past the vocabulary, where the output has some: zeros)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col + e >= p.V) v[e] = 0.0f;
      }
      store_chunk<F32>(p.y, row * p.ldy, col, p.cols_out, v);
    }
    if (PEN && p.drafts && r + 1 < r1) {
      __syncthreads();
      count_path(~0u);
    }
  }
}

template <bool F32, int IT, bool PEN, bool BIAS, bool MASK>
hipError_t launch_as(const LogitsParams& p, hipStream_t s) {
  constexpr int C = kThreads * 8 * IT;
  const int bytes = (PEN + BIAS) * C * 4 + (PEN && p.drafts ? tree_lds_bytes(p.rows) + p.rows * 4 : 0);
  const int64_t grid = (int64_t)((p.cols_out + C - 1) / C) * ((p.rows + p.group - 1) / p.group) * p.batch;
  logits_kernel<F32, IT, PEN, BIAS, MASK><<<(unsigned)grid, kThreads, bytes, s>>>(p);
  return hipGetLastError();
}

template <bool F32, int IT>
hipError_t launch_rules(const LogitsParams& p, hipStream_t s) {
  const int rules = (p.history ? 4 : 0) + (p.bias_tokens ? 2 : 0) + (p.mask ? 1 : 0);
  switch (rules) {
    case 1: return launch_as<F32, IT, false, false, true>(p, s);
    case 2: return launch_as<F32, IT, false, true, false>(p, s);
    case 3: return launch_as<F32, IT, false, true, true>(p, s);
    case 4: return launch_as<F32, IT, true, false, false>(p, s);
    case 5: return launch_as<F32, IT, true, false, true>(p, s);
    case 6: return launch_as<F32, IT, true, true, false>(p, s);
    case 7: return launch_as<F32, IT, true, true, true>(p, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

void choose_logits(LogitsParams& p) { p.group = p.rows; }

hipError_t launch_logits(const LogitsParams& p, hipStream_t s) {
  if (p.drafts && p.rows > kMaxTree) return hipErrorInvalidValue;
  return p.f32 ? launch_rules<true, 2>(p, s) : launch_rules<false, 2>(p, s);
}

}  // namespace byoc
