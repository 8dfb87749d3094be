// Which tokens of a tree of drafts each of them sees, from their parents (ckv_tree_sees).
//
// Tokens in blocks of 64: a wave finds each token's path inside its block by doubling (six exchanges: what is known of a token's path, and of the path
// of where that ends, joined), as a word of bits and the token in an earlier block that the path leaves to. A token's words are then those of
// the blocks that its path runs through, at most one step a block. A parent is an earlier token, so a path ends and runs through blocks in order.
#include "ckv_pages.h"

namespace ckv {

constexpr int kTreeThreads = 256;

__global__ void __launch_bounds__(kTreeThreads) tree_sees_kernel(const int32_t *parent, const int32_t *start, uint64_t *sees, int32_t *positions, int n) {
  __shared__ uint64_t s_bits[kMostDrafts];
  __shared__ int s_leaves[kMostDrafts];
  const int chunks = (n + kTreeThreads - 1) / kTreeThreads, b = blockIdx.x / chunks, first = blockIdx.x % chunks * kTreeThreads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, words = (n + 63) / 64;
  const int last = min(first + kTreeThreads, n) - 1;  // token whose path is the last one that is looked at
  for (int block = wave; block <= last / 64; block += kTreeThreads / kWave) {
    const int i = block * 64 + lane;
    const int p = i < n ? parent[(size_t)b * n + i] : -1;
    const bool has = p >= 0 && p < i;
    int to = has && p >= block * 64 ? p - block * 64 : -1;  // where the known part of the path goes on
    int root = lane;                                        // the last token of that part
    const int leaves = has && p < block * 64 ? p : -1;
    uint64_t bits = 1ull << lane;
#pragma unroll
    for (int round = 0; round < 6; ++round) {
      const int from = to >= 0 ? to : lane;
      const uint64_t more = __shfl((unsigned long long)bits, from);
      const int further = __shfl(to, from), end = __shfl(root, from);
      if (to >= 0) {
        bits |= more;
        root = end;
        to = further;
      }
    }
    const int out = __shfl(leaves, root);
    s_bits[i] = bits;
    s_leaves[i] = out;
  }
  __syncthreads();
  const int i = first + threadIdx.x;
  if (i >= n) return;
  uint64_t *to = sees + ((size_t)b * n + i) * words;
  int at = i, depth = -1;
  for (int w = words - 1; w >= 0; --w) {
    uint64_t bits = 0;
    if (at >= 0 && at >> 6 == w) {
      bits = s_bits[at];
      at = s_leaves[at];
      depth += __popcll(bits);
    }
    to[w] = bits;
  }
  if (positions) positions[(size_t)b * n + i] = (int32_t)((uint32_t)start[b] + (uint32_t)depth);
}

hipError_t launch_tree_sees(int batch, int n, const int32_t *parent, const int32_t *start, uint64_t *sees, int32_t *positions, hipStream_t stream) {
  const unsigned chunks = (unsigned)(n + kTreeThreads - 1) / kTreeThreads;
  hipLaunchKernelGGL(tree_sees_kernel, dim3(batch * chunks), dim3(kTreeThreads), 0, stream, parent, start, sees, positions, n);
  return hipGetLastError();
}

}  // namespace ckv
