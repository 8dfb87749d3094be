// Attention of new tokens over lists of pages (ckv_paged_attention).
//
// Columns: the queries of a (batch element, KV head), G * i + head, so that neighbours see nearly the same rows and a row is read once
// for all heads of a group. A workgroup takes a tile of columns, 32 per wave, and sweeps the rows that the last of them sees, in stages
// of 64 (bf16) or 32 (f32) rows that go from memory to LDS without registers between and are read by all of its waves.
// Rows x queries (32 x 32 matrix tiles, 16 or 2 components at a time) leaves a lane with 16 logits of one column, whose running
// maximum and sum stay in the lane but for one exchange with the other half of the wave, and which are the operand of the second product as
// they lie: the contraction over rows may be permuted if both operands agree, so V's operand takes the rows in the order that the
// logits have. V lies in LDS as it does in memory and is transposed on its way into registers.
// LDS images are swizzled in units that one cycle reads (16 bytes of eight rows of K, 32 bytes of four rows of V).
//
// What a token does not see must not touch its result even if it is infinite or NaN, and zero times infinity is NaN: where a sweep leaves
// something that is not finite, the workgroup sweeps again, with V's finite components only, and twice more for where its
// infinite and NaN ones are.
#include <type_traits>

#include "ckv_pages.h"

namespace ckv {

struct PagedArgs {
  const char *q, *k, *v;
  int64_t qs[3];       // BYTES between batch elements, query heads, tokens
  PageLists lists;
  char *out;
  int64_t os[3];       // BYTES, as qs
  float *lse;          // [Bz][Hq][n] natural log, or null
  float *part;         // [unit][column tile][chunk][column of the tile][d]: weighted sums of V
  float2 *stats;       // [unit][column tile][chunk][column of the tile]: running maximum (log2), sum
  int Hq, Hkv, G, n, n_rows, n_chunks, col_tiles;
  int workgroups;
  float scale2;        // softmax scale * log2(e)
};

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_p;
typedef __attribute__((ext_vector_type(16))) float f32x16_p;
typedef __attribute__((ext_vector_type(4))) float f32x4_p;
typedef __attribute__((ext_vector_type(4))) short s16x4_p;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_p;

constexpr int kXcdsP = 8;  // accelerator dies of the part; workgroup i of a launch runs on die i % 8

typedef __attribute__((address_space(1))) const void global_t;
typedef __attribute__((address_space(3))) void lds_t;
// 16 bytes a lane from `from` to lds + 16 * lane; lds is the same for the wave.
__device__ __forceinline__ void load_to_lds(const char *from, char *lds) {
  __builtin_amdgcn_global_load_lds((global_t *)from, (lds_t *)lds, 16, 0, 0);
}
// All of the wave's loads are there.
__device__ __forceinline__ void wait_lds_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }
// Four 16-bit words a lane, transposed among 16 lanes: lane i gets word i % 4 of what lanes i / 4, 4 + i / 4, 8 + i / 4, 12 + i / 4 read.
__device__ __forceinline__ u32x2_p read_transposed(const char *lds) {
  typedef __attribute__((address_space(3))) s16x4_p lds_words;
  return __builtin_bit_cast(u32x2_p, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_words *)lds));
}

template <int DT, int DH>
struct Stage {
  static constexpr int ESIZE = DT == CKV_BF16 ? 2 : 4;
  static constexpr int ROW = DH * ESIZE;               // bytes
  static constexpr int CHUNKS = ROW / 16;              // 16-byte pieces of a row
  static constexpr int KEYS = DT == CKV_BF16 ? 64 : 32;
  static constexpr int BYTES = KEYS * ROW;             // of K, and of V
  static constexpr int BLOCKS = KEYS / 32;
  static constexpr int ROWS_PER_LOAD = 1024 / ROW;     // a wave's load of 16 bytes a lane
  // place of piece c of row r
  static __device__ __forceinline__ int k_piece(int r, int c) { return c ^ (r & 7); }
  static __device__ __forceinline__ int v_piece(int r, int c) {
    if (DT != CKV_BF16) return c;
    return c ^ (2 * (ROW == 128 ? (r >> 1) & 3 : r & 3));
  }
};
constexpr int stage_keys(bool bf16) { return bf16 ? 64 : 32; }

// The rows that the tile's columns see, and how its chunks share them: whole stages.
struct TileRange {
  int cols;        // columns of the tile that exist
  int end;         // rows that the last of them sees
  int stages, per_chunk;
};
__device__ __forceinline__ TileRange tile_range(const PagedArgs &a, int unit, int tile, int tile_cols, int keys) {
  TileRange t;
  const int count = new_rows(a.lists, unit, a.n), length = max(a.lists.length[unit], 0);
  t.cols = min(a.G * count - tile * tile_cols, tile_cols);
  const int last = (tile * tile_cols + t.cols - 1) / a.G;
  t.end = t.cols > 0 ? min(max(length - count + last + 1, 0), a.n_rows) : 0;
  t.stages = (t.end + keys - 1) / keys;
  t.per_chunk = max(1, (t.stages + a.n_chunks - 1) / a.n_chunks);
  return t;
}

// Sum, maximum over the two lanes (l, l ^ 32) that share a column.
template <class Op>
__device__ __forceinline__ float over_halves(float x, Op op) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// Eight (bf16) or four (f32) contraction indexes of each half of the wave.
template <int DT>
__device__ __forceinline__ void mma_piece(f32x16_p &acc, const u32x4_d &x, const u32x4_d &y) {
  if (DT == CKV_BF16) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_p, x), __builtin_bit_cast(bf16x8_p, y), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[e]), __uint_as_float(y[e]), acc, 0, 0, 0);
  }
}

// How a second sweep takes V's components: the finite ones only, or ones where there is an infinity of one sign or a NaN.
enum VMode { kUp, kDown, kFinite };
template <int DT>
__device__ __forceinline__ uint32_t v_word(uint32_t x, int mode) {
  if (DT == CKV_BF16) {
    uint32_t out = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t b = (x >> (16 * h)) & 0xffffu;
      const bool finite = (b & 0x7f80u) != 0x7f80u, nan = !finite && (b & 0x7fu);
      const bool marked = !finite && (nan || (mode == kUp) == !(b & 0x8000u));
      out |= (mode == kFinite ? (finite ? b : 0u) : (marked ? 0x3f80u : 0u)) << (16 * h);
    }
    return out;
  }
  const bool finite = (x & 0x7f800000u) != 0x7f800000u, nan = !finite && (x & 0x7fffffu);
  const bool marked = !finite && (nan || (mode == kUp) == !(x & 0x80000000u));
  return mode == kFinite ? (finite ? x : 0u) : (marked ? 0x3f800000u : 0u);
}

// Workgroup `id` of a launch: XCD id % 8 gets a contiguous part of the work, so that the workgroups that read the same
// rows at the same time share an L2.
__device__ __forceinline__ int work_item(int id, int total) {
  const int xcd = id % kXcdsP, at = id / kXcdsP, each = total / kXcdsP, more = total % kXcdsP;
  return xcd * each + min(xcd, more) + at;
}

template <int DT, int DH, int WAVES>
__global__ void __launch_bounds__(WAVES *kWave, 2) paged_tile_kernel(PagedArgs a) {
  typedef Stage<DT, DH> S;
  constexpr int TILE = WAVES * 32;
  constexpr int STEPS = S::CHUNKS / 2;     // pieces of a row per half of the wave
  constexpr int DTILES = DH / 32;
  constexpr int LOADS = S::BYTES / 1024 / WAVES;  // of K per wave and stage, and of V
  static_assert(LOADS * WAVES * 1024 == S::BYTES, "whole loads");
  __shared__ __align__(1024) char s_k[2][S::BYTES];
  __shared__ __align__(1024) char s_v[2][S::BYTES];
  __shared__ int s_bad, s_undefined;

  int at = work_item(blockIdx.x, a.workgroups);
  const int chunk = at % a.n_chunks;
  at /= a.n_chunks;
  const int tile = a.col_tiles - 1 - at % a.col_tiles, unit = at / a.col_tiles;  // the longest first
  const int b = unit / a.Hkv, g = unit % a.Hkv;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 31, half = lane >> 5;
  const TileRange range = tile_range(a, unit, tile, TILE, S::KEYS);
  if (range.cols <= 0) return;
  const int first_stage = chunk * range.per_chunk, last_stage = min(first_stage + range.per_chunk, range.stages);
  const bool single = a.n_chunks == 1;
  if (first_stage >= last_stage && !single) return;  // the merge reads the chunks that have stages

  const int local = wave * 32 + m, col = tile * TILE + local;
  const bool valid = local < range.cols;
  const int token = col / a.G, h = g * a.G + col % a.G;
  const int count = new_rows(a.lists, unit, a.n), length = max(a.lists.length[unit], 0);
  const int limit = valid ? min(max(length - count + token + 1, 0), a.n_rows) : 0;  // rows that the column sees
  // of the wave: its first column sees the fewest rows, the last that exists the most
  const int sees_least = __builtin_amdgcn_readfirstlane(limit);
  const int last_local = min(range.cols, wave * 32 + 32) - 1;
  const int sees_most = last_local < wave * 32 ? 0 : min(max(length - count + (tile * TILE + last_local) / a.G + 1, 0), a.n_rows);

  u32x4_d qf[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    qf[s] = u32x4_d{0u, 0u, 0u, 0u};
    if (valid) qf[s] = *reinterpret_cast<const u32x4_d *>(a.q + b * a.qs[0] + h * a.qs[1] + token * a.qs[2] + (2 * s + half) * 16);
  }

  const int32_t *list = a.lists.table + b * a.lists.table_b + g * a.lists.table_h;
  const char *kb = a.k + g * a.lists.ks[1], *vb = a.v + g * a.lists.vs[1];
  const int in_page = (1 << a.lists.shift) - 1;
  if (threadIdx.x == 0) s_bad = s_undefined = 0;
  __syncthreads();

  // Rows behind the end are the last one again; a page that is not in the pool is page 0 (they weigh nothing).
  auto fetch = [&](int stage, int buf) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int block = wave * LOADS + j, row = block * S::ROWS_PER_LOAD + lane / S::CHUNKS, piece = lane % S::CHUNKS;
      const int key = min(stage * S::KEYS + row, range.end - 1);
      int page = list[key >> a.lists.shift];
      if ((unsigned)page >= (unsigned)a.lists.n_pages) {
        page = 0;
        s_bad = 1;
      }
      const int64_t r = key & in_page;
      // k_piece and v_piece are their own inverses
      load_to_lds(kb + page * a.lists.ks[0] + r * a.lists.ks[2] + S::k_piece(row, piece) * 16, s_k[buf] + block * 1024);
      load_to_lds(vb + page * a.lists.vs[0] + r * a.lists.vs[2] + S::v_piece(row, piece) * 16, s_v[buf] + block * 1024);
    }
  };

  float top = -INFINITY, sum = 0.0f;  // of the column; this half's share of the sum
  f32x16_p acc[DTILES];               // component 32 t + 8 (r / 4) + 4 half + r % 4 of the column
  // CAREFUL: V's components as `mode` says
  auto sweep = [&](auto careful, int mode) {
    constexpr bool CAREFUL = decltype(careful)::value;
    top = -INFINITY;
    sum = 0.0f;
#pragma unroll
    for (int t = 0; t < DTILES; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[t][r] = 0.0f;
    if (first_stage < last_stage) fetch(first_stage, 0);
    for (int stage = first_stage; stage < last_stage; ++stage) {
      const int buf = (stage - first_stage) & 1;
      wait_lds_loads();
      __syncthreads();  // the stage is there, and the other buffer has been read
      if (stage + 1 < last_stage) fetch(stage + 1, buf ^ 1);
      const int base = stage * S::KEYS;
      if (base >= sees_most) continue;
      const bool bad = s_bad;
      f32x16_p z[S::BLOCKS];
#pragma unroll
      for (int k = 0; k < S::BLOCKS; ++k) {
#pragma unroll
        for (int r = 0; r < 16; ++r) z[k][r] = 0.0f;
        const int row = 32 * k + m;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
          mma_piece<DT>(z[k], *reinterpret_cast<const u32x4_d *>(s_k[buf] + row * S::ROW + S::k_piece(row, 2 * s + half) * 16), qf[s]);
      }
      if (bad || base + S::KEYS > sees_least) {
#pragma unroll
        for (int k = 0; k < S::BLOCKS; ++k)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = base + 32 * k + 8 * (r / 4) + 4 * half + r % 4;
            bool seen = key < limit;
            if (bad && seen) seen = (unsigned)list[key >> a.lists.shift] < (unsigned)a.lists.n_pages;
            if (!seen) z[k][r] = -INFINITY;
          }
      }
      float mx = z[0][0];
#pragma unroll
      for (int k = 0; k < S::BLOCKS; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, z[k][r]);
      mx = over_halves(mx, [](float x, float y) { return fmaxf(x, y); }) * a.scale2;
      if (__any(mx > top)) {
        const float now = fmaxf(top, mx);
        const float keep = exp2f(top - (now == -INFINITY ? 0.0f : now));
        sum *= keep;
#pragma unroll
        for (int t = 0; t < DTILES; ++t) acc[t] *= keep;
        top = now;
      }
      const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
      for (int k = 0; k < S::BLOCKS; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float seen = CAREFUL && z[k][r] != -INFINITY ? 1.0f : 0.0f;
          z[k][r] = __builtin_amdgcn_exp2f(fmaf(z[k][r], a.scale2, -ref));
          sum += z[k][r];
          if (CAREFUL && mode != kFinite) z[k][r] = seen;
        }
#pragma unroll
      for (int k = 0; k < S::BLOCKS; ++k) {
        if constexpr (DT == CKV_BF16) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            u32x4_d w;  // the column's weights of rows 16 j + 4 half + (0..3) and eight further on
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack_bf16(z[k][8 * j + 2 * e], z[k][8 * j + 2 * e + 1]);
#pragma unroll
            for (int t = 0; t < DTILES; ++t) {
              u32x4_d x;
#pragma unroll
              for (int p = 0; p < 2; ++p) {
                // 16 lanes read four rows of 16 components and get a component's four rows each
                const int row = 32 * k + 16 * j + 8 * p + 4 * half + (lane & 15) / 4;
                const int byte = 64 * t + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
                const u32x2_p two = read_transposed(s_v[buf] + row * S::ROW + S::v_piece(row, byte / 16) * 16 + byte % 16);
                x[2 * p] = two[0];
                x[2 * p + 1] = two[1];
              }
              if (CAREFUL)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = v_word<DT>(x[e], mode);
              mma_piece<DT>(acc[t], x, w);
            }
          }
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int row = 32 * k + 8 * (r / 4) + 4 * half + r % 4;
#pragma unroll
            for (int t = 0; t < DTILES; ++t) {
              uint32_t x = *reinterpret_cast<const uint32_t *>(s_v[buf] + row * S::ROW + (32 * t + m) * 4);
              if (CAREFUL) x = v_word<DT>(x, mode);
              acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x), z[k][r], acc[t], 0, 0, 0);
            }
          }
        }
      }
    }
  };
  sweep(std::false_type{}, kFinite);

  bool undefined = false;
#pragma unroll
  for (int t = 0; t < DTILES; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) undefined |= !(fabsf(acc[t][r]) < INFINITY);
  if (undefined && valid) s_undefined = 1;
  __syncthreads();
  if (s_undefined) {  // V has components that are not finite, or the logits have: the same for all waves, as there are barriers in the sweeps
    uint64_t up = 0, down = 0;
    for (int mode = kUp; mode <= kFinite; ++mode) {
      __syncthreads();  // the buffers have been read
      sweep(std::true_type{}, mode);
#pragma unroll
      for (int t = 0; t < DTILES; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint64_t bit = 1ull << (16 * t + r);
          if (mode == kUp) up |= acc[t][r] > 0.0f ? bit : 0;
          else if (mode == kDown) down |= acc[t][r] > 0.0f ? bit : 0;
          else if ((up | down) & bit) acc[t][r] += !(up & bit) ? -INFINITY : !(down & bit) ? INFINITY : NAN;
        }
    }
  }
  sum = over_halves(sum, [](float x, float y) { return x + y; });
  if (!valid) return;

  if (single) {
    char *to = a.out + b * a.os[0] + h * a.os[1] + token * a.os[2];
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int t = 0; t < DTILES; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = 32 * t + 8 * r + 4 * half;
        if (DT == CKV_BF16)
          *reinterpret_cast<uint2 *>(to + 2 * d) = make_uint2(pack_bf16(acc[t][4 * r] * inv, acc[t][4 * r + 1] * inv),
                                                             pack_bf16(acc[t][4 * r + 2] * inv, acc[t][4 * r + 3] * inv));
        else
          *reinterpret_cast<f32x4_p *>(to + 4 * d) =
              f32x4_p{acc[t][4 * r] * inv, acc[t][4 * r + 1] * inv, acc[t][4 * r + 2] * inv, acc[t][4 * r + 3] * inv};
      }
    if (a.lse && half == 0)
      a.lse[((size_t)b * a.Hq + h) * a.n + token] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
    return;
  }
  const size_t row = (((size_t)unit * a.col_tiles + tile) * a.n_chunks + chunk) * TILE + local;
  float *to = a.part + row * DH;
#pragma unroll
  for (int t = 0; t < DTILES; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *reinterpret_cast<f32x4_p *>(to + 32 * t + 8 * r + 4 * half) =
          f32x4_p{acc[t][4 * r], acc[t][4 * r + 1], acc[t][4 * r + 2], acc[t][4 * r + 3]};
  if (half == 0) a.stats[row] = make_float2(top, sum);
}

// Chunks of a column, in their order. A thread takes four components of one column.
constexpr int kMergeThreads = 256;
template <int DT, int DH>
__global__ void __launch_bounds__(kMergeThreads) paged_merge_kernel(PagedArgs a, int tile_cols) {
  constexpr int KEYS = stage_keys(DT == CKV_BF16), LPC = DH / 4, COLS = kMergeThreads / LPC;
  const int cols = a.G * a.n, blocks = (cols + COLS - 1) / COLS;
  const int unit = blockIdx.x / blocks, col = blockIdx.x % blocks * COLS + threadIdx.x / LPC, c = threadIdx.x % LPC * 4;
  const int b = unit / a.Hkv, g = unit % a.Hkv;
  if (col >= a.G * new_rows(a.lists, unit, a.n)) return;
  const int tile = col / tile_cols, token = col / a.G, h = g * a.G + col % a.G;
  const TileRange range = tile_range(a, unit, tile, tile_cols, KEYS);
  const int chunks = (range.stages + range.per_chunk - 1) / range.per_chunk;
  const size_t first = ((size_t)unit * a.col_tiles + tile) * a.n_chunks * tile_cols + col % tile_cols;
  float top = -INFINITY;
  for (int i = 0; i < chunks; ++i) {
    top = fmaxf(top, a.stats[first + (size_t)i * tile_cols].x);
  }
  const float ref = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f;
  f32x4_p num = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i = 0; i < chunks; ++i) {
    const size_t row = first + (size_t)i * tile_cols;
    const float2 st = a.stats[row];
    const f32x4_p x = *reinterpret_cast<const f32x4_p *>(a.part + row * DH + c);
    const float f = exp2f(st.x - ref);
    sum = fmaf(st.y, f, sum);
#pragma unroll
    for (int e = 0; e < 4; ++e) num[e] = fabsf(x[e]) < INFINITY ? fmaf(x[e], f, num[e]) : num[e] + x[e];  // infinity weighs in, however little
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  num *= inv;
  char *to = a.out + b * a.os[0] + h * a.os[1] + token * a.os[2];
  if (DT == CKV_BF16) *reinterpret_cast<uint2 *>(to + 2 * c) = make_uint2(pack_bf16(num[0], num[1]), pack_bf16(num[2], num[3]));
  else *reinterpret_cast<f32x4_p *>(to + 4 * c) = num;
  if (a.lse && c == 0) a.lse[((size_t)b * a.Hq + h) * a.n + token] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
constexpr int kTileWaves = 4;

PagedPlan plan_paged(const Shape &s, int n_rows) {
  PagedPlan p;
  const int keys = stage_keys(s.esize == 2);
  const int64_t units = (int64_t)s.Bz * s.Hkv, cols = (int64_t)s.G * s.T;
  p.tile_cols = kTileWaves * 32;
  p.col_tiles = (int)((cols + p.tile_cols - 1) / p.tile_cols);
  const int64_t tiles = units * p.col_tiles, stages = (n_rows + keys - 1) / keys;
  int64_t chunks = 2 * kComputeUnits / tiles;
  if (chunks > (stages + 3) / 4) chunks = (stages + 3) / 4;
  if (chunks > 64) chunks = 64;
  if (chunks < 1) chunks = 1;
  p.n_chunks = (int)chunks;
  p.workgroups = tiles * chunks;
  p.workspace_bytes = chunks == 1 ? 0 : (size_t)p.workgroups * p.tile_cols * (s.d + 2) * sizeof(float);
  return p;
}

template <int DT, int DH>
static void launch_paged_of(const PagedArgs &a, const PagedPlan &plan, int units, hipStream_t stream) {
  hipLaunchKernelGGL((paged_tile_kernel<DT, DH, kTileWaves>), dim3((unsigned)plan.workgroups), dim3(kTileWaves * kWave), 0, stream, a);
  if (plan.n_chunks > 1) {
    constexpr int COLS = kMergeThreads / (DH / 4);
    const unsigned blocks = (unsigned)(a.G * a.n + COLS - 1) / COLS;
    hipLaunchKernelGGL((paged_merge_kernel<DT, DH>), dim3(units * blocks), dim3(kMergeThreads), 0, stream, a, plan.tile_cols);
  }
}

PageLists page_lists(const Shape &s, const ckv_pages *pages, const int32_t *table, const int32_t *length, const int32_t *count) {
  PageLists l;
  l.table = table;
  l.length = length;
  l.count = count;
  l.table_b = pages->table_stride[0];
  l.table_h = pages->table_stride[1];
  for (int i = 0; i < 3; ++i) {
    l.ks[i] = pages->k_stride[i] * s.esize;
    l.vs[i] = pages->v_stride[i] * s.esize;
  }
  l.shift = __builtin_ctz((unsigned)pages->page_rows);
  l.n_pages = pages->n_pages;
  l.capacity = pages->max_pages * pages->page_rows;
  return l;
}

hipError_t launch_paged_attention(const ckv_params *p, const Shape &s, const PagedPlan &plan, const ckv_pages *pages, const void *q,
                                  const void *k_pages, const void *v_pages, const int32_t *table, const int32_t *length,
                                  const int32_t *count, int n_rows, void *out, const int64_t *out_stride, float *lse, char *ws,
                                  hipStream_t stream) {
  PagedArgs a;
  a.q = static_cast<const char *>(q);
  a.k = static_cast<const char *>(k_pages);
  a.v = static_cast<const char *>(v_pages);
  a.out = static_cast<char *>(out);
  const int64_t dense[3] = {(int64_t)s.Hq * s.T * s.d, (int64_t)s.T * s.d, s.d};
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = p->q_stride[i] * s.esize;
    a.os[i] = (out_stride ? out_stride[i] : dense[i]) * s.esize;
  }
  a.lists = page_lists(s, pages, table, length, count);
  a.lse = lse;
  a.part = reinterpret_cast<float *>(ws);
  a.stats = reinterpret_cast<float2 *>(a.part + (plan.n_chunks > 1 ? (size_t)plan.workgroups * plan.tile_cols * s.d : 0));
  a.Hq = s.Hq; a.Hkv = s.Hkv; a.G = s.G;
  a.n = s.T;
  a.n_rows = n_rows;
  a.n_chunks = plan.n_chunks;
  a.col_tiles = plan.col_tiles;
  a.workgroups = (int)plan.workgroups;
  a.scale2 = s.scale * kLog2e;
  const int units = s.Bz * s.Hkv;
  if (p->dtype == CKV_BF16) {
    if (s.d == 128) launch_paged_of<CKV_BF16, 128>(a, plan, units, stream);
    else launch_paged_of<CKV_BF16, 64>(a, plan, units, stream);
  } else {
    if (s.d == 128) launch_paged_of<CKV_F32, 128>(a, plan, units, stream);
    else launch_paged_of<CKV_F32, 64>(a, plan, units, stream);
  }
  return hipGetLastError();
}

}  // namespace ckv
