// Paths of a tree of drafted tokens: token j's parent is one of the tokens before it,
// or -1 for a child of the last accepted token; anything else counts as -1, so that
// every path ends.
#pragma once

#include "device_common.h"
#include "limits.h"

namespace byoc {

// LDS of the paths of n tokens: `words` words a token (bit k: token k is on its path,
// the token itself included), and the tokens' next ancestors.
struct TreePaths {
  uint32_t* bits;
  int* up;
  int words;
  __device__ __forceinline__ uint32_t word(int j, int w) const { return bits[j * words + w]; }
};
__host__ __device__ constexpr int tree_words(int n) { return (n + 31) / 32; }
__host__ __device__ constexpr int tree_lds_bytes(int n) { return n * (tree_words(n) + 1) * 4; }

// Formed by all NT threads of a workgroup, each path twice as long with every round
// (a token's path up to its next ancestor joins that one's), so that the longest
// chain takes 8 rounds.  Ends with a barrier.
template <int NT>
__device__ __forceinline__ TreePaths form_paths(const int* parents, int n, uint32_t* lds) {
  const TreePaths t{lds, (int*)lds + n * tree_words(n), tree_words(n)};
  constexpr int W = tree_words(kMaxTree);
  bool more = false;
  for (int j = threadIdx.x; j < n; j += NT) {
    const int p = parents[j], u = p >= 0 && p < j ? p : -1;
    t.up[j] = u;
    more |= u >= 0;
    for (int w = 0; w < t.words; ++w) t.bits[j * t.words + w] = j >> 5 == w ? 1u << (j & 31) : 0u;
  }
  while (__syncthreads_or(more)) {
    more = false;
    for (int j0 = 0; j0 < n; j0 += NT) {
      const int j = j0 + threadIdx.x, u = j < n ? t.up[j] : -1;
      uint32_t got[W];
      int next = -1;
      if (u >= 0) {
        next = t.up[u];
#pragma unroll
        for (int w = 0; w < W; ++w) got[w] = w < t.words ? t.bits[u * t.words + w] : 0u;
      }
      __syncthreads();
      if (u >= 0) {
        t.up[j] = next;
        more |= next >= 0;
#pragma unroll
        for (int w = 0; w < W; ++w)
          if (w < t.words) t.bits[j * t.words + w] |= got[w];
      }
      if (j0 + NT < n) __syncthreads();
    }
  }
  return t;
}

}  // namespace byoc
