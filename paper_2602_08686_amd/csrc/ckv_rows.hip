// New rows on their way into a cache: RMS norm of every head, position rotation, and the place in the pages.
//
// Bound by memory: every row read once and written once, 2 * d * e bytes of it; on the way there, the address arithmetic costs more than the
// rotation. So a workgroup takes a few tokens of a sequence with some of their KV heads, and first makes, in LDS, what all lanes
// of its rows need: the cosines and sines of each token's angles (the same for all its heads) and, a thread for each (token, KV
// head), where its rows come from and go to, page numbers looked up. Then 8 or 16 lanes take a (token, KV head): the key, the value and the
// group's queries go through registers, eight components a lane, all their loads in flight together. A lane of the rotated
// front holds four components and their four partners, so that no lane needs another's: halves (c, c + rot/2) lie in two pieces of
// four, neighbours in eight consecutive ones. Sums of squares cross the row's lanes as operands of the additions. Rows without
// norm and rotation (values; keys that the retention step kept) are copied as bits.
//
// Measured, bf16, 32/8 heads of 128, norm and rotation: 32768 tokens 137 us, 4.9 TB/s of reads and writes, where a copy of 320 MiB reaches 5.4; up to
// 4099 tokens of two sequences into pages, with their queries 43 us; one token of each of 16 sequences 5 us, a launch.
// Angles: position * inv_freq / (2 pi) in fp64, off by less than 2^-51 of itself (2^-31 of a turn a million turns away), and without
// its whole turns to fp32.
#include <type_traits>

#include "ckv_pages.h"

namespace ckv {

struct RowsArgs {
  const char *q, *k, *v;           // q or k may be null (no such rows); v null: dense outputs
  int64_t qs[3], ks[3], vs[3];     // BYTES between batch elements, heads, tokens
  const void *q_weight, *k_weight; // [d] or null
  const int32_t *positions;        // [Bz][n]
  const float *inv_freq;           // [rot / 2]
  char *q_out, *k_out, *v_out;     // dense [Bz][H][n][d]; with pages k_out and v_out are the pools
  PageLists lists;                 // without pages only `count` of it
  int Hq, Hkv, G, n;
  int rot, norm;
  float eps;
  int tokens, token_blocks;        // tokens of a workgroup (a power of two), workgroups along a sequence
  int heads;                       // KV heads of a workgroup (grid.y of them)
};

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_r;

constexpr int kRowThreads = 256;
constexpr int kMostTokens = 8;     // tokens of a workgroup
constexpr int kMostHeads = kRowThreads / kMostTokens;  // KV heads: a thread for every (token, head)

// Four components as they lie in memory; as fp32; and back: to the nearest, ties to even, the one rounding of a row's way.
template <int DT>
struct Four {
  typedef typename std::conditional<DT == CKV_BF16, u32x2_r, u32x4_d>::type raw_t;
};
template <int DT>
__device__ __forceinline__ typename Four<DT>::raw_t load_four(const char *p) {
  return *reinterpret_cast<const typename Four<DT>::raw_t *>(p);
}
template <int DT>
__device__ __forceinline__ void to_floats(const typename Four<DT>::raw_t &raw, float *x) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    x[e] = __uint_as_float(DT != CKV_BF16 ? raw[DT != CKV_BF16 ? e : 0] : e % 2 ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16);
}
template <int DT>
__device__ __forceinline__ typename Four<DT>::raw_t from_floats(const float *x) {
  typename Four<DT>::raw_t raw;
  if constexpr (DT == CKV_BF16) {
    raw = u32x2_r{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) raw[e] = __float_as_uint(x[e]);
  }
  return raw;
}

enum RowForm { kCopied, kHalves, kNeighbours };  // what happens to keys and queries: nothing, or norm and rotation in these pairs

// Eight components of a row in a lane, at `at0` and `at1` bytes (four each), or as they are.
template <int DT, int DH, int FORM>
struct LaneRow {
  static constexpr bool NEIGHBOURS = FORM == kNeighbours;
  typename Four<DT>::raw_t lo, hi;
  __device__ __forceinline__ void load(const char *row, int at0, int at1) {
    lo = load_four<DT>(row + at0);
    hi = load_four<DT>(row + at1);
  }
  // all lanes of the row take part
  __device__ __forceinline__ void change(bool norm, float eps, const float (&w)[8], bool turned, const float2 (&turn)[4]) {
    float x[8];
    to_floats<DT>(lo, &x[0]);
    to_floats<DT>(hi, &x[4]);
    if (norm) {
      float sq = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sq = fmaf(x[e], x[e], sq);
      sq = row_sum<DH / 8>(sq);
      const float f = __builtin_amdgcn_rsqf(fmaf(sq, 1.0f / DH, eps));  // one unit of the last place
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] * f * w[e];
    }
    if (turned) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // the pair's two components: (e, 4 + e) of the pieces, or neighbours
        float &p = NEIGHBOURS ? x[2 * e] : x[e], &p2 = NEIGHBOURS ? x[2 * e + 1] : x[4 + e];
        const float y = p, y2 = p2;
        p = y * turn[e].x - y2 * turn[e].y;
        p2 = y2 * turn[e].x + y * turn[e].y;
      }
    }
    lo = from_floats<DT>(&x[0]);
    hi = from_floats<DT>(&x[4]);
  }
  __device__ __forceinline__ void store(char *row, int at0, int at1) const {
    *reinterpret_cast<typename Four<DT>::raw_t *>(row + at0) = lo;
    *reinterpret_cast<typename Four<DT>::raw_t *>(row + at1) = hi;
  }
};
template <int DT, int DH>
struct LaneRow<DT, DH, kCopied> {
  static constexpr int WORDS = DT == CKV_BF16 ? 1 : 2;
  u32x4_d x[WORDS];
  __device__ __forceinline__ void load(const char *row, int at0, int) {
#pragma unroll
    for (int w = 0; w < WORDS; ++w) x[w] = *reinterpret_cast<const u32x4_d *>(row + at0 + 16 * w);
  }
  __device__ __forceinline__ void change(bool, float, const float (&)[8], bool, const float2 (&)[4]) {}
  __device__ __forceinline__ void store(char *row, int at0, int) const {
#pragma unroll
    for (int w = 0; w < WORDS; ++w) *reinterpret_cast<u32x4_d *>(row + at0 + 16 * w) = x[w];
  }
};

// PAGED: keys and values go into pages, else keys are dense and there are no values.
template <int DT, int DH, int FORM, bool PAGED>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(RowsArgs a) {
  constexpr bool TRANSFORM = FORM != kCopied;
  constexpr int ESIZE = DT == CKV_BF16 ? 2 : 4, ROW = DH * ESIZE;
  constexpr int LPR = DH / 8;                 // lanes of a row
  constexpr int ABREAST = kRowThreads / LPR;  // (token, KV head)s at a time
  constexpr int Q = 4;                        // queries whose loads are in flight together
  __shared__ float2 s_turn[kMostTokens][TRANSFORM ? DH / 2 : 1];  // cosine and sine
  struct Way {                                // BYTES from the tensors' starts
    int64_t q, k, v, q_out, k_out, v_out;
    int32_t here, placed;                     // the row is one of the call's; k_out and v_out are in the pools
  };
  __shared__ Way s_way[kRowThreads];
  const int b = blockIdx.x / a.token_blocks, first = (blockIdx.x % a.token_blocks) * a.tokens;
  const int g0 = blockIdx.y * a.heads, heads = min(a.heads, a.Hkv - g0), ways = a.tokens * heads;
  const int sub = threadIdx.x % LPR, slot = threadIdx.x / LPR;

  if ((int)threadIdx.x < ways) {
    const int i = first + threadIdx.x % a.tokens, g = g0 + threadIdx.x / a.tokens, unit = b * a.Hkv + g, h = g * a.G;
    const int count = new_rows(a.lists, unit, a.n);
    Way w;
    w.here = i < min(count, a.n);
    w.placed = w.here;
    w.q = b * a.qs[0] + h * a.qs[1] + i * a.qs[2];
    w.k = b * a.ks[0] + g * a.ks[1] + i * a.ks[2];
    w.v = b * a.vs[0] + g * a.vs[1] + i * a.vs[2];
    w.q_out = (((int64_t)b * a.Hq + h) * a.n + i) * ROW;
    w.k_out = ((int64_t)unit * a.n + i) * ROW;
    w.v_out = 0;
    if (PAGED && w.here) {
      const int at = max(a.lists.length[unit], 0) - count + i;
      w.placed = at >= 0 && at < a.lists.capacity;
      if (w.placed) {
        const int page = a.lists.table[b * a.lists.table_b + g * a.lists.table_h + (at >> a.lists.shift)], row = at & ((1 << a.lists.shift) - 1);
        w.placed = (unsigned)page < (unsigned)a.lists.n_pages;
        w.k_out = in_pool(a.lists.ks, page, g, row);
        w.v_out = in_pool(a.lists.vs, page, g, row);
      }
    }
    s_way[threadIdx.x] = w;
  }
  if (TRANSFORM && a.rot > 0) {
    const int half = a.rot / 2, tokens = min(a.tokens, a.n - first);
    for (int i = threadIdx.x; i < tokens * half; i += kRowThreads) {
      const int t = i / half, c = i - t * half;
      const double turns = (double)a.positions[(size_t)b * a.n + first + t] * (double)a.inv_freq[c] * 0.15915494309189535;
      float2 cs;
      sincospif(2.0f * (float)(turns - rint(turns)), &cs.y, &cs.x);
      s_turn[t][c] = cs;
    }
  }
  __syncthreads();

  // pieces of the lane: bytes from the row's start
  const bool turned = TRANSFORM && sub < a.rot / 8;
  const bool apart = turned && FORM == kHalves;
  const int at0 = apart ? 4 * sub * ESIZE : 8 * sub * ESIZE;
  const int at1 = apart ? (a.rot / 2 + 4 * sub) * ESIZE : at0 + 4 * ESIZE;
  float qw[8], kw[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) qw[e] = kw[e] = 1.0f;
  if (TRANSFORM && a.norm && a.q_weight) {
    to_floats<DT>(load_four<DT>(static_cast<const char *>(a.q_weight) + at0), &qw[0]);
    to_floats<DT>(load_four<DT>(static_cast<const char *>(a.q_weight) + at1), &qw[4]);
  }
  if (TRANSFORM && a.norm && a.k_weight) {
    to_floats<DT>(load_four<DT>(static_cast<const char *>(a.k_weight) + at0), &kw[0]);
    to_floats<DT>(load_four<DT>(static_cast<const char *>(a.k_weight) + at1), &kw[4]);
  }

  // A (token, KV head)'s rows.
  struct Rows {
    LaneRow<DT, DH, FORM> key, query[Q];
    LaneRow<DT, DH, kCopied> value;
  };
  const int queries = a.q ? a.G : 0;
  auto load = [&](Rows &rows, int i) CKV_INLINE {
    if (i >= ways || !s_way[i].here) return;
    const Way &w = s_way[i];
    if (a.k) rows.key.load(a.k + w.k, at0, at1);
    if (PAGED) rows.value.load(a.v + w.v, 8 * sub * ESIZE, 0);
    const char *from = a.q + w.q;
#pragma unroll
    for (int h = 0; h < Q; ++h)
      if (h < queries) rows.query[h].load(from + h * a.qs[1], at0, at1);
  };
  auto finish = [&](Rows &rows, int i) CKV_INLINE {
    const Way &w = s_way[i];
    if (!w.here) return;  // a row's lanes all go on or none does
    const int64_t to_step = (int64_t)a.n * ROW;
    const char *from = a.q + w.q;
    char *to = a.q_out + w.q_out;
    float2 turn[4];
    if (turned) {
#pragma unroll
      for (int e = 0; e < 4; ++e) turn[e] = s_turn[i % a.tokens][4 * sub + e];
    }
    if (a.k) {
      rows.key.change(a.norm, a.eps, kw, turned, turn);
      if (w.placed) rows.key.store(a.k_out + w.k_out, at0, at1);
    }
    if (PAGED && w.placed) rows.value.store(a.v_out + w.v_out, 8 * sub * ESIZE, 0);
    for (int h0 = 0; h0 < queries; h0 += Q) {
#pragma unroll
      for (int h = 0; h < Q; ++h) {
        if (h0 + h < queries) {
          rows.query[h].change(a.norm, a.eps, qw, turned, turn);
          rows.query[h].store(to + (h0 + h) * to_step, at0, at1);
          if (h0 + Q + h < queries) rows.query[h].load(from + (h0 + Q + h) * a.qs[1], at0, at1);
        }
      }
    }
  };
  // Dense bf16 rows: the next (token, KV head)'s are on their way while these are worked on (a 32k prompt 145 -> 137 us). Into pages, and
  // in f32, the registers that this takes cost more than it brings (a chunk of 4k tokens 46.5 -> 49.9).
  constexpr bool AHEAD = !PAGED && DT == CKV_BF16;
  Rows even, odd;
  if (AHEAD) load(even, slot);
  for (int i = slot; i < ways; i += (AHEAD ? 2 : 1) * ABREAST) {
    if (!AHEAD) {
      load(even, i);
      finish(even, i);
      continue;
    }
    load(odd, i + ABREAST);
    finish(even, i);
    if (i + ABREAST >= ways) break;
    load(even, i + 2 * ABREAST);
    finish(odd, i + ABREAST);
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
template <int DT, int DH, int FORM>
static void launch_rows_as(const RowsArgs &a, dim3 grid, bool paged, hipStream_t stream) {
  if (paged) hipLaunchKernelGGL((rows_kernel<DT, DH, FORM, true>), grid, dim3(kRowThreads), 0, stream, a);
  else hipLaunchKernelGGL((rows_kernel<DT, DH, FORM, false>), grid, dim3(kRowThreads), 0, stream, a);
}
template <int DT, int DH>
static void launch_rows_of(const RowsArgs &a, dim3 grid, RowForm form, bool paged, hipStream_t stream) {
  if (form == kHalves) launch_rows_as<DT, DH, kHalves>(a, grid, paged, stream);
  else if (form == kNeighbours) launch_rows_as<DT, DH, kNeighbours>(a, grid, paged, stream);
  else launch_rows_as<DT, DH, kCopied>(a, grid, paged, stream);
}

// pages null: dense outputs and no values.
hipError_t launch_rows(const ckv_params *p, const Shape &s, const ckv_rotation *rotation, const ckv_pages *pages, const void *q,
                       const void *k, const void *v, const int32_t *positions, const float *inv_freq, const void *q_weight,
                       const void *k_weight, const int32_t *table, const int32_t *length, const int32_t *count, void *q_out, void *k_out,
                       void *v_out, hipStream_t stream) {
  RowsArgs a;
  a.q = static_cast<const char *>(q);
  a.k = static_cast<const char *>(k);
  a.v = static_cast<const char *>(v);
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = p->q_stride[i] * s.esize;
    a.ks[i] = p->k_stride[i] * s.esize;
    a.vs[i] = p->v_stride[i] * s.esize;
  }
  a.q_weight = q_weight;
  a.k_weight = k_weight;
  a.positions = positions;
  a.inv_freq = inv_freq;
  a.q_out = static_cast<char *>(q_out);
  a.k_out = static_cast<char *>(k_out);
  a.v_out = static_cast<char *>(v_out);
  if (pages) a.lists = page_lists(s, pages, table, length, count);
  else a.lists = PageLists();
  a.lists.count = count;
  a.Hq = s.Hq; a.Hkv = s.Hkv; a.G = s.G;
  a.n = s.T;
  a.rot = rotation ? rotation->rot_dim : 0;
  a.norm = rotation ? rotation->norm : 0;
  a.eps = rotation ? rotation->norm_eps : 0.0f;
  // Long calls: a few tokens a workgroup, so that the angles are made once for all heads. Short ones: a token's heads over several workgroups, each
  // of which makes the angles again. us, one token a workgroup / these: 32768 tokens 161 / 137, batch 2 of 1024 12.0 / 10.3; all heads in one / these:
  // batch 32 of 4 tokens into pages 7.2 / 6.3.
  const int64_t tokens = (int64_t)s.Bz * s.T;
  a.tokens = 1;
  while (a.tokens < kMostTokens && 2 * a.tokens <= s.T && tokens / (2 * a.tokens) >= 4 * kComputeUnits) a.tokens *= 2;
  a.token_blocks = (s.T + a.tokens - 1) / a.tokens;
  const int64_t blocks = (int64_t)s.Bz * a.token_blocks;
  a.heads = s.Hkv < kMostHeads ? s.Hkv : kMostHeads;
  while (a.heads > 1 && blocks * ((s.Hkv + a.heads - 1) / a.heads) < kComputeUnits) a.heads = (a.heads + 1) / 2;
  const dim3 grid((unsigned)blocks, (unsigned)((s.Hkv + a.heads - 1) / a.heads));
  const RowForm form = a.rot == 0 && !a.norm ? kCopied : a.rot > 0 && rotation->pairing == CKV_PAIR_NEIGHBOURS ? kNeighbours : kHalves;
  if (p->dtype == CKV_BF16) {
    if (s.d == 128) launch_rows_of<CKV_BF16, 128>(a, grid, form, pages != nullptr, stream);
    else launch_rows_of<CKV_BF16, 64>(a, grid, form, pages != nullptr, stream);
  } else {
    if (s.d == 128) launch_rows_of<CKV_F32, 128>(a, grid, form, pages != nullptr, stream);
    else launch_rows_of<CKV_F32, 64>(a, grid, form, pages != nullptr, stream);
  }
  return hipGetLastError();
}

}  // namespace ckv
