// New rows on their way into a cache: RMS norm of every head, position rotation, and the place in the pages.
//
// Bound by memory: every row read once and written once, 2 * d * e bytes of it. A workgroup takes a few tokens of a sequence: it makes
// the cosines and sines of their angles once, in LDS (a token's angles are those of all its heads), and its heads' rows go through
// registers, eight components a lane. A lane of the rotated front holds four components and their four partners, so that no lane needs
// another's: halves (c, c + rot/2) lie in two pieces of four, neighbours in eight consecutive ones. Sums of squares cross the row's
// lanes as operands of the additions. Rows without norm and rotation (values; keys that the retention step kept) are copied as bits.
//
// Angles: position * inv_freq / (2 pi) in fp64, off by less than 2^-51 of itself (2^-31 of a turn a million turns away), and without
// its whole turns to fp32.
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
  int q_rows, k_rows, rows;        // rows of a token: queries, keys, and all (values behind the keys)
  int tokens, token_blocks;        // tokens of a workgroup, workgroups along a sequence
  int split_rows;                  // rows of a token that one workgroup takes (grid.y of them)
};

constexpr int kRowThreads = 256;
constexpr int kMostTokens = 8;     // tokens of a workgroup

// Eight components in two pieces of four, as fp32.
template <int DT>
__device__ __forceinline__ void load_four(const char *p, float *x) {
  if (DT == CKV_BF16) {
    const uint2 raw = *reinterpret_cast<const uint2 *>(p);
    x[0] = __uint_as_float(raw.x << 16);
    x[1] = __uint_as_float(raw.x & 0xffff0000u);
    x[2] = __uint_as_float(raw.y << 16);
    x[3] = __uint_as_float(raw.y & 0xffff0000u);
  } else {
    const uint4 raw = *reinterpret_cast<const uint4 *>(p);
    x[0] = __uint_as_float(raw.x);
    x[1] = __uint_as_float(raw.y);
    x[2] = __uint_as_float(raw.z);
    x[3] = __uint_as_float(raw.w);
  }
}
template <int DT>
__device__ __forceinline__ void store_four(char *p, const float *x) {
  if (DT == CKV_BF16) {  // the one rounding: to the nearest, ties to even
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
  } else {
    *reinterpret_cast<uint4 *>(p) =
        make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
}

enum RowForm { kCopied, kHalves, kNeighbours };  // what happens to keys and queries: nothing, or norm and rotation in these pairs
// U: rows whose loads a lane has in flight.
// PAGED: keys and values go into pages, else keys are dense and there are no values.
template <int DT, int DH, int FORM, bool PAGED, int U>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(RowsArgs a) {
  constexpr bool TRANSFORM = FORM != kCopied, NEIGHBOURS = FORM == kNeighbours;
  constexpr int ESIZE = DT == CKV_BF16 ? 2 : 4, ROW = DH * ESIZE;
  constexpr int LPR = DH / 8;                 // lanes of a row
  constexpr int ABREAST = kRowThreads / LPR;  // rows at a time
  constexpr int PIECE = 4 * ESIZE;
  __shared__ float2 s_turn[kMostTokens][TRANSFORM ? DH / 2 : 1];  // cosine and sine
  const int b = blockIdx.x / a.token_blocks, first = (blockIdx.x % a.token_blocks) * a.tokens;
  const int tokens = min(a.tokens, a.n - first);
  const int r0 = blockIdx.y * a.split_rows, split = min(a.split_rows, a.rows - r0);
  const int sub = threadIdx.x % LPR, slot = threadIdx.x / LPR;

  if (TRANSFORM && a.rot > 0) {
    const int half = a.rot / 2;
    for (int i = threadIdx.x; i < tokens * half; i += kRowThreads) {
      const int t = i / half, c = i % half;
      const double turns = (double)a.positions[(size_t)b * a.n + first + t] * (double)a.inv_freq[c] * 0.15915494309189535;
      float2 cs;
      sincospif(2.0f * (float)(turns - rint(turns)), &cs.y, &cs.x);
      s_turn[t][c] = cs;
    }
    __syncthreads();
  }

  // pieces of the lane: bytes from the row's start
  const bool turned = TRANSFORM && sub < a.rot / 8;
  const bool apart = turned && !NEIGHBOURS;
  const int at0 = apart ? 4 * sub * ESIZE : 8 * sub * ESIZE;
  const int at1 = apart ? (a.rot / 2 + 4 * sub) * ESIZE : at0 + PIECE;
  float qw[8], kw[8];
  if (TRANSFORM) {
#pragma unroll
    for (int e = 0; e < 8; ++e) qw[e] = kw[e] = 1.0f;
    if (a.norm && a.q_weight) {
      load_four<DT>(static_cast<const char *>(a.q_weight) + at0, &qw[0]);
      load_four<DT>(static_cast<const char *>(a.q_weight) + at1, &qw[4]);
    }
    if (a.norm && a.k_weight) {
      load_four<DT>(static_cast<const char *>(a.k_weight) + at0, &kw[0]);
      load_four<DT>(static_cast<const char *>(a.k_weight) + at1, &kw[4]);
    }
  }

  // rows of the workgroup in the order (token, row of the token), ABREAST of them at a time
  int t = slot / split, r = slot % split;
  while (t < tokens) {
    float x[U][8];
    u32x4_d raw[U][ESIZE / 2];
    char *to[U];       // where the row goes, or null
    bool here[U], keys[U], copied[U];
    int token[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      to[u] = nullptr;
      here[u] = keys[u] = false;
      copied[u] = !TRANSFORM;
      token[u] = t;
      if (t < tokens) {
        const int row = r0 + r, i = first + t;
        const bool query = row < a.q_rows;
        keys[u] = !query && row < a.q_rows + a.k_rows;
        copied[u] = !TRANSFORM || (!query && !keys[u]);
        const int h = query ? row : row - a.q_rows - (keys[u] ? 0 : a.k_rows), g = query ? h / a.G : h, unit = b * a.Hkv + g;
        const int count = new_rows(a.lists, unit, a.n);
        here[u] = i < count;
        if (here[u]) {
          const char *src = query ? a.q + b * a.qs[0] + h * a.qs[1] + i * a.qs[2]
                          : keys[u] ? a.k + b * a.ks[0] + h * a.ks[1] + i * a.ks[2]
                                    : a.v + b * a.vs[0] + h * a.vs[1] + i * a.vs[2];
          if (copied[u]) {
#pragma unroll
            for (int w = 0; w < ESIZE / 2; ++w) raw[u][w] = *reinterpret_cast<const u32x4_d *>(src + sub * 8 * ESIZE + 16 * w);
          } else {
            load_four<DT>(src + at0, &x[u][0]);
            load_four<DT>(src + at1, &x[u][4]);
          }
          if (query) {
            to[u] = a.q_out + (((size_t)b * a.Hq + h) * a.n + i) * ROW;
          } else if (!PAGED) {
            to[u] = a.k_out + ((size_t)unit * a.n + i) * ROW;
          } else {
            const int at = max(a.lists.length[unit], 0) - count + i;
            if (at >= 0 && at < a.lists.capacity) {
              const int page = a.lists.table[b * a.lists.table_b + g * a.lists.table_h + (at >> a.lists.shift)];
              const int in_page = at & ((1 << a.lists.shift) - 1);
              if ((unsigned)page < (unsigned)a.lists.n_pages)
                to[u] = keys[u] ? a.k_out + in_pool(a.lists.ks, page, g, in_page) : a.v_out + in_pool(a.lists.vs, page, g, in_page);
            }
          }
        }
      }
      r += ABREAST;
      while (r >= split) {
        r -= split;
        ++t;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (TRANSFORM && a.norm) {
        float sq = 0.0f;
        if (here[u] && !copied[u]) {
#pragma unroll
          for (int e = 0; e < 8; ++e) sq = fmaf(x[u][e], x[u][e], sq);
        }
        sq = row_sum<LPR>(sq);  // a row's lanes are all here or none is
        if (here[u] && !copied[u]) {
          const float f = 1.0f / sqrtf(sq * (1.0f / DH) + a.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[u][e] = x[u][e] * f * (keys[u] ? kw[e] : qw[e]);
        }
      }
      if (!to[u]) continue;
      if (copied[u]) {
#pragma unroll
        for (int w = 0; w < ESIZE / 2; ++w) *reinterpret_cast<u32x4_d *>(to[u] + sub * 8 * ESIZE + 16 * w) = raw[u][w];
        continue;
      }
      if (turned) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 cs = s_turn[token[u]][4 * sub + e];
          // the pair's two components: (e, 4 + e) of the pieces, or neighbours
          float &p = NEIGHBOURS ? x[u][2 * e] : x[u][e], &p2 = NEIGHBOURS ? x[u][2 * e + 1] : x[u][4 + e];
          const float y = p, y2 = p2;
          p = y * cs.x - y2 * cs.y;
          p2 = y2 * cs.x + y * cs.y;
        }
      }
      store_four<DT>(to[u] + at0, &x[u][0]);
      store_four<DT>(to[u] + at1, &x[u][4]);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
template <int DT, int DH, int FORM>
static void launch_rows_as(const RowsArgs &a, dim3 grid, bool paged, hipStream_t stream) {
  if (paged) hipLaunchKernelGGL((rows_kernel<DT, DH, FORM, true, 4>), grid, dim3(kRowThreads), 0, stream, a);
  else hipLaunchKernelGGL((rows_kernel<DT, DH, FORM, false, 4>), grid, dim3(kRowThreads), 0, stream, a);
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
  a.q_rows = q ? s.Hq : 0;
  a.k_rows = k ? s.Hkv : 0;
  a.rows = a.q_rows + a.k_rows + (v ? s.Hkv : 0);
  // Long calls: a few tokens a workgroup, so that the angles are made once for all heads. Short ones: a token's rows over
  // several workgroups, each of which makes the angles again.
  const int abreast = kRowThreads / (s.d / 8);
  const int64_t tokens = (int64_t)s.Bz * s.T;
  a.tokens = 1;
  while (a.tokens < kMostTokens && tokens / (2 * a.tokens) >= 4 * kComputeUnits) a.tokens *= 2;
  a.token_blocks = (s.T + a.tokens - 1) / a.tokens;
  const int64_t blocks = (int64_t)s.Bz * a.token_blocks;
  int splits = 1;
  while (blocks * splits < 2 * kComputeUnits && splits * abreast < a.rows) ++splits;
  a.split_rows = (a.rows + splits - 1) / splits;
  splits = (a.rows + a.split_rows - 1) / a.split_rows;
  const dim3 grid((unsigned)blocks, (unsigned)splits);
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
