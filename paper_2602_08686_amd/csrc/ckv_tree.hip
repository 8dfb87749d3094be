// Which tokens of a tree of drafts each of them sees, from their parents (ckv_tree_sees).
//
// Tokens in blocks of 64: a wave finds each token's path inside its block by doubling (six exchanges: what is known of a token's path, and of the path
// of where that ends, joined), as a word of bits and the token in an earlier block that the path leaves to. A token's words are then those of
// the blocks that its path runs through, at most one step a block. A parent is an earlier token, so a path ends and runs through blocks in order.
#include "ckv_pages.h"
#include <ckv_dma.h>

namespace ckv {

constexpr int kTreeThreads = 512;
constexpr int kTreeStage = 16;  // words of a token that leave LDS together: 128 bytes

// MOST: tokens of a sequence that there is room for. The words go to memory by way of LDS, a token's side by side; written by the lane that finds them, a
// store touched 64 lines (64 sequences of 1000 tokens 9.4 us, now 6.4). Above 1024 tokens a call takes 9.2 us for 16 sequences of 2000, 18.2 for 16 of 4096 (34 MB
// written: 6.6) and 14.9 for one of 4096, whose eight workgroups each find the paths of all tokens in front of theirs.
template <int MOST>
__global__ void __launch_bounds__(kTreeThreads) tree_sees_kernel(const int32_t *parent, const int32_t *start, uint64_t *sees, int32_t *positions, int n) {
  __shared__ uint64_t s_bits[MOST];
  __shared__ int s_leaves[MOST];
  __shared__ uint64_t s_words[kTreeThreads / kWave][kTreeStage][kWave + 1];
  const int chunks = (n + kTreeThreads - 1) / kTreeThreads, b = blockIdx.x / chunks, first = blockIdx.x % chunks * kTreeThreads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, words = (n + 63) / 64;
  const int last = min(first + kTreeThreads, n) - 1;  // token whose path is the last one that is looked at
  const int from0 = positions ? start[b] : 0;
  auto parent_of = [&](int i) CKV_INLINE { return i < n ? parent[(size_t)b * n + i] : -1; };
  int next = parent_of(wave * 64 + lane);
  for (int block = wave; block <= last / 64; block += kTreeThreads / kWave) {
    const int i = block * 64 + lane, p = next;
    next = parent_of(i + kTreeThreads);
    const bool has = p >= 0 && p < i;
    int to = has && p >= block * 64 ? p - block * 64 : -1;  // where the known part of the path goes on
    int root = lane;                                        // the last token of that part
    const int leaves = has && p < block * 64 ? p : -1;
    uint64_t bits = 1ull << lane;
    for (int round = 0; round < 6 && __any(to >= 0); ++round) {
      const int from = to >= 0 ? to : lane;
      const uint64_t more = __shfl((unsigned long long)bits, from);
      const int further = __shfl(to * 256 | root, from);
      if (to >= 0) {
        bits |= more;
        root = further & 255;
        to = further >> 8;
      }
    }
    const int out = __shfl(leaves, root);
    s_bits[i] = bits;
    s_leaves[i] = out;
  }
  __syncthreads();
  const int i = first + threadIdx.x, tokens = min(n - (first + wave * kWave), kWave);
  if (tokens <= 0) return;
  uint64_t *to = sees + ((size_t)b * n + first + wave * kWave) * words;  // of the wave's first token
  int at = i < n ? i : -1, depth = -1;
  for (int w0 = (words - 1) / kTreeStage * kTreeStage; w0 >= 0; w0 -= kTreeStage) {
    const int some = min(words - w0, kTreeStage);
    for (int w = some - 1; w >= 0; --w) {
      uint64_t bits = 0;
      if (at >= 0 && at >> 6 == w0 + w) {
        bits = s_bits[at];
        at = s_leaves[at];
        depth += __popcll(bits);
      }
      s_words[wave][w][lane] = bits;
    }
    wait_lds_reads();
    const int aside = some <= 1 ? 1 : some <= 2 ? 2 : some <= 4 ? 4 : some <= 8 ? 8 : 16, w = lane % aside;
    for (int t = lane / aside; t < tokens; t += kWave / aside)
      if (w < some) to[(size_t)t * words + w0 + w] = s_words[wave][w][t];
    wait_lds_reads();
  }
  if (positions && i < n) positions[(size_t)b * n + i] = (int32_t)((uint32_t)from0 + (uint32_t)depth);
}

int64_t tree_workgroups(int batch, int n) { return (int64_t)batch * ((n + kTreeThreads - 1) / kTreeThreads); }

hipError_t launch_tree_sees(int batch, int n, const int32_t *parent, const int32_t *start, uint64_t *sees, int32_t *positions, hipStream_t stream) {
  const dim3 grid((unsigned)tree_workgroups(batch, n));
  if (n <= 1024) hipLaunchKernelGGL(tree_sees_kernel<1024>, grid, dim3(kTreeThreads), 0, stream, parent, start, sees, positions, n);
  else hipLaunchKernelGGL(tree_sees_kernel<kMostDrafts>, grid, dim3(kTreeThreads), 0, stream, parent, start, sees, positions, n);
  return hipGetLastError();
}

}  // namespace ckv
