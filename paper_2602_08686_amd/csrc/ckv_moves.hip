// Rows that move inside their pages (ckv_paged_compact) and pages that are copied (ckv_pages_copy).
#include "ckv_pages.h"
#include <ckv_dma.h>

namespace ckv {

// ---------------------------------------------------------------------------------------------
// Rows
// ---------------------------------------------------------------------------------------------
// In place: row r of the moved ones comes from idx[r] >= r (ascending numbers, none twice), so what is written for r holds no source of a later
// row, and the sources that it does hold are those of rows up to r. Reads may run ahead of writes as far as they like; a write waits for the
// reads of its own round and the earlier ones, which a workgroup that takes a list's rows in order has behind a barrier a round. The pieces of a row are
// independent, so keys, values and parts of rows go to workgroups of their own. Short lists are a chain of four trips to memory (lengths, numbers, pages, rows):
// seven accepted rows of 16 sequences, 8 heads 3.6 us, up to 544 kept rows of 32 lists 6.7; long ones are bound by what a few workgroups a list have in
// flight (bf16, 8 lists, all of 16384 of 32768 rows 82 us, 134 MB read and written at 1.6 TB/s) or by memory (f32, 48 lists, up to 9362 of 14438 rows 169 us, 692 MB
// at 4.1 TB/s). Figures with "up to", and those below, are of calls that keep between half of it and all, three quarters on average.
struct CompactArgs {
  PageLists lists;  // count null: all rows of a list
  char *k, *v;
  const int32_t *idx, *kept;
  int64_t idx_b, idx_h;
  int32_t *length_out;
  int cap, Hkv;
  int row_pieces;  // of 16 bytes of a row
  int pieces;      // of a row's keys and values that a workgroup takes: a power of two
  int splits;      // workgroups of a list
};

constexpr int kRowsOfOne = 5, kRowsOfMany = 4;  // of a thread in a round, where one round does, and where more may be needed

// LONG: more than one round may be needed, and three of them are side by side: a row's number in the list, the pages of where it is and where it goes, and the
// row itself, each a trip to memory behind the other. us, one round after the other / side by side: 16384 of 32768 rows, 8 heads 86 / 64, 10931 of 20114,
// 5 lists 52 / 31. (For a single round the registers of the others cost more than they bring: 544 rows, 128 lists 13.2 / 16.0.)
template <bool LONG>
__global__ void __launch_bounds__(1024, LONG ? 4 : 8) compact_rows_kernel(CompactArgs a) {
  constexpr int AHEAD = LONG ? kRowsOfMany : kRowsOfOne;
  const int unit = blockIdx.x / a.splits, slice = blockIdx.x % a.splits, b = unit / a.Hkv, g = unit % a.Hkv;
  const int length = max(a.lists.length[unit], 0);
  const int count = a.lists.count ? min(max(a.lists.count[unit], 0), length) : length, first = length - count;
  const int stay = min(max(a.kept[unit], 0), min(count, a.cap));
  if (slice == 0 && threadIdx.x == 0) a.length_out[unit] = first + stay;
  const int m = min(stay, min(a.lists.capacity, INT32_MAX - (1 << 16)) - first);  // rows behind the list's pages go nowhere; room for the rounds ahead
  const int piece = slice * a.pieces + threadIdx.x % a.pieces, rows = blockDim.x / a.pieces, mine = threadIdx.x / a.pieces;
  const bool values = piece >= a.row_pieces;
  const int64_t s_page = values ? a.lists.vs[0] : a.lists.ks[0], s_row = values ? a.lists.vs[2] : a.lists.ks[2];
  char *base = (values ? a.v + g * a.lists.vs[1] : a.k + g * a.lists.ks[1]) + (piece - (values ? a.row_pieces : 0)) * 16;
  const int32_t *list = a.lists.table + b * a.lists.table_b + g * a.lists.table_h, *idx = a.idx + b * a.idx_b + g * a.idx_h;
  const int in_page = (1 << a.lists.shift) - 1;
  struct Pages {
    int from, to, row;  // row: in the list, of where it is; -1: it does not move
  };
  auto row_of = [&](int round, int j) CKV_INLINE { return (round * AHEAD + j) * rows + mine; };
  auto find = [&](int round, int (&from)[AHEAD]) CKV_INLINE {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) from[j] = row_of(round, j) < m ? idx[row_of(round, j)] : -1;
  };
  auto turn = [&](int round, const int (&from)[AHEAD], Pages (&p)[AHEAD]) CKV_INLINE {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int to = first + row_of(round, j), row = first + from[j];
      const bool moves = from[j] >= 0 && from[j] < count && row != to && row < a.lists.capacity && to < a.lists.capacity;
      p[j] = Pages{-1, -1, -1};
      if (moves) p[j] = Pages{list[row >> a.lists.shift], list[to >> a.lists.shift], row};
    }
  };
  auto read = [&](Pages (&p)[AHEAD], u32x4_d (&x)[AHEAD]) CKV_INLINE {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if ((unsigned)p[j].from >= (unsigned)a.lists.n_pages || (unsigned)p[j].to >= (unsigned)a.lists.n_pages) p[j].row = -1;
      x[j] = u32x4_d{0u, 0u, 0u, 0u};
      if (p[j].row >= 0) x[j] = *reinterpret_cast<const u32x4_d *>(base + p[j].from * s_page + (p[j].row & in_page) * s_row);
    }
  };
  int from[AHEAD];
  Pages here[AHEAD], next[AHEAD];
  u32x4_d x[AHEAD];
  find(0, from);
  turn(0, from, here);
  if (LONG) find(1, from);
  read(here, x);
  if (LONG) {
    turn(1, from, next);
    find(2, from);
  }
  for (int round = 0; LONG ? round * AHEAD * rows < m : round < 1; ++round) {
    u32x4_d ahead[AHEAD];
    Pages then[AHEAD];
    if (LONG) {
      read(next, ahead);
      turn(round + 2, from, then);
      find(round + 3, from);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) asm volatile("" : "+v"(x[j]));  // this round's rows are there; the next one's may be on their way
    __syncthreads();
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (here[j].row >= 0) *reinterpret_cast<u32x4_d *>(base + here[j].to * s_page + ((first + row_of(round, j)) & in_page) * s_row) = x[j];
      if (LONG) {
        x[j] = ahead[j];
        here[j] = next[j];
        next[j] = then[j];
      }
    }
  }
}

hipError_t launch_compact(const Shape &s, const ckv_pages *pages, const int32_t *table, const int32_t *length, const int32_t *count,
                          const int32_t *idx, const int64_t *idx_stride, int cap, const int32_t *kept, void *k_pages, void *v_pages,
                          int32_t *length_out, hipStream_t stream) {
  CompactArgs a;
  a.lists = page_lists(s, pages, table, length, count);
  a.k = static_cast<char *>(k_pages);
  a.v = static_cast<char *>(v_pages);
  a.idx = idx;
  a.kept = kept;
  a.idx_b = idx_stride ? idx_stride[0] : (int64_t)s.Hkv * cap;
  a.idx_h = idx_stride ? idx_stride[1] : cap;
  a.length_out = length_out;
  a.cap = cap;
  a.Hkv = s.Hkv;
  a.row_pieces = s.d * s.esize / 16;
  // Short lists by a workgroup each; others in parts of 128 bytes of a row, or 64 where long lists leave most CUs idle (us, 128 / 64 bytes: 10931 of 20114
  // rows, 5 lists 45 / 31, 16384 of 32768, 8 lists 73 / 64, 8192 of 32768, 32 lists 62.6 / 66.5).
  a.pieces = (int64_t)cap * 2 * a.row_pieces <= 1024 ? 2 * a.row_pieces : 8;
  if (a.pieces == 8 && cap > 1024 && (int64_t)s.Bz * s.Hkv * a.row_pieces / 4 <= kComputeUnits / 4) a.pieces = 4;
  a.splits = 2 * a.row_pieces / a.pieces;
  static_assert(kMostUnits * 16ll * 1024 < 1ll << 32, "a list has 16 workgroups of 1024 threads at most, a launch fewer than 2^32 threads");
  int threads = 1024;
  while (threads > 64 && (int64_t)cap * a.pieces <= threads / 2) threads /= 2;
  const dim3 grid((unsigned)(s.Bz * s.Hkv * a.splits));
  if (cap > kRowsOfOne * (threads / a.pieces)) hipLaunchKernelGGL(compact_rows_kernel<true>, grid, dim3(threads), 0, stream, a);
  else hipLaunchKernelGGL(compact_rows_kernel<false>, grid, dim3(threads), 0, stream, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Pages
// ---------------------------------------------------------------------------------------------
// A workgroup takes 32 KiB of a pair, a thread eight pieces of 16 bytes, all read before the first is written. Memory bound: bf16, 1000 pages of 64 rows of 8 heads
// 106.5 us, 4.9 TB/s read and written (a plain copy of a gigabyte 5.1); 16 pages of 16 rows 3.3 us, a launch.
struct CopyArgs {
  char *k, *v;
  const int32_t *copy;
  int64_t ks[3], vs[3];  // BYTES between pages, KV heads, rows
  int n_pages, shift;    // log2(page_rows)
  int heads, piece_shift;  // log2(pieces of 16 bytes of a row)
  int total, parts;      // pieces of a pair, keys and values; workgroups of a pair
};
constexpr int kCopyThreads = 256, kCopyAhead = 8;

__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(CopyArgs a) {
  const int pair = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const int src = a.copy[2 * (size_t)pair], dst = a.copy[2 * (size_t)pair + 1];
  if ((unsigned)src >= (unsigned)a.n_pages || (unsigned)dst >= (unsigned)a.n_pages || src == dst) return;
  u32x4_d x[kCopyAhead];
  char *to[kCopyAhead];
#pragma unroll
  for (int j = 0; j < kCopyAhead; ++j) {
    const int64_t at = ((int64_t)part * kCopyAhead + j) * kCopyThreads + threadIdx.x;
    const int i = (int)(at < a.total ? at : a.total - 1);
    const int piece = i & ((1 << a.piece_shift) - 1), row = i >> a.piece_shift & ((1 << a.shift) - 1), h = i >> (a.piece_shift + a.shift);
    const bool values = h >= a.heads;
    const int64_t in_page = piece * 16 + (values ? (h - a.heads) * a.vs[1] + row * a.vs[2] : h * a.ks[1] + row * a.ks[2]);
    x[j] = *reinterpret_cast<const u32x4_d *>((values ? a.v + src * a.vs[0] : a.k + src * a.ks[0]) + in_page);
    to[j] = (values ? a.v + dst * a.vs[0] : a.k + dst * a.ks[0]) + in_page;
  }
#pragma unroll
  for (int j = 0; j < kCopyAhead; ++j)
    if (((int64_t)part * kCopyAhead + j) * kCopyThreads + threadIdx.x < a.total) *reinterpret_cast<u32x4_d *>(to[j]) = x[j];
}

// Heads of a page in memory.
static int heads_of(const Shape &s, const ckv_pages *pages) { return pages->k_stride[1] == 0 && pages->v_stride[1] == 0 ? 1 : s.Hkv; }
static int64_t pieces_of(const Shape &s, const ckv_pages *pages) {
  return (int64_t)2 * heads_of(s, pages) * pages->page_rows * (s.d * s.esize / 16);
}
int64_t copy_workgroups(const Shape &s, const ckv_pages *pages, int n) {
  const int64_t pieces = pieces_of(s, pages), each = kCopyThreads * kCopyAhead;
  return pieces > INT32_MAX ? INT64_MAX : n * ((pieces + each - 1) / each);
}

hipError_t launch_pages_copy(const Shape &s, const ckv_pages *pages, const int32_t *copy, int n, void *k_pages, void *v_pages, hipStream_t stream) {
  CopyArgs a;
  a.k = static_cast<char *>(k_pages);
  a.v = static_cast<char *>(v_pages);
  a.copy = copy;
  for (int i = 0; i < 3; ++i) {
    a.ks[i] = pages->k_stride[i] * s.esize;
    a.vs[i] = pages->v_stride[i] * s.esize;
  }
  a.n_pages = pages->n_pages;
  a.shift = __builtin_ctz((unsigned)pages->page_rows);
  a.heads = heads_of(s, pages);
  a.piece_shift = __builtin_ctz((unsigned)(s.d * s.esize / 16));
  a.total = (int)pieces_of(s, pages);
  a.parts = (int)(copy_workgroups(s, pages, 1));
  hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)copy_workgroups(s, pages, n)), dim3(kCopyThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ckv
