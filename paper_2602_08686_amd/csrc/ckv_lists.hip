// Which lists have which pages: lists that share pages (ckv_pages_fork), get some (ckv_pages_reserve) and give them back (ckv_pages_free).
//
// A page's count says how many entries name it, a bit per page whether any does: the free pages are the zero bits, found 32 at a word. What several
// entries do to a page at once are additions and bits set or cleared, in any order the same; who gets which page goes by the order of the entries.
#include "ckv_pages.h"
#include <ckv_dma.h>

namespace ckv {

struct ListArgs {
  int32_t *table;
  int64_t table_b, table_h;
  int32_t *refs;
  uint32_t *taken;
  int Hkv, heads, lists;  // heads: lists of a batch element
  int n_pages, shift, max_pages;
};

static ListArgs list_args(const ckv_lists *l, int32_t *table, int32_t *refs, uint32_t *taken) {
  ListArgs a;
  a.table = table;
  a.table_b = l->table_stride[0];
  a.table_h = l->table_stride[1];
  a.refs = refs;
  a.taken = taken;
  a.Hkv = l->n_kv_heads;
  a.heads = l->table_stride[1] == 0 ? 1 : l->n_kv_heads;
  a.lists = l->batch * a.heads;
  a.n_pages = l->n_pages;
  a.shift = __builtin_ctz((unsigned)l->page_rows);
  a.max_pages = l->max_pages;
  return a;
}

// Atomic at device scope: past the first-level caches.
template <class T>
__device__ __forceinline__ T add_across(T *p, T v) { return __scoped_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE); }
__device__ __forceinline__ void min_across(int32_t *p, int32_t v) { __scoped_atomic_fetch_min(p, v, __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE); }
__device__ __forceinline__ void take_page(const ListArgs &a, int p) {
  __scoped_atomic_fetch_or(a.taken + (p >> 5), 1u << (p & 31), __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE);
}
__device__ __forceinline__ bool in_pool(const ListArgs &a, int p) { return (unsigned)p < (unsigned)a.n_pages; }
// One entry less names the page. (A count that says none did keeps saying so.)
__device__ __forceinline__ void release_page(const ListArgs &a, int p) {
  const int before = add_across(a.refs + p, -1);
  if (before == 1) __scoped_atomic_fetch_and(a.taken + (p >> 5), ~(1u << (p & 31)), __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE);
  else if (before < 1) add_across(a.refs + p, 1);
}
__device__ __forceinline__ int32_t *list_of(const ListArgs &a, int l) { return a.table + l / a.heads * a.table_b + l % a.heads * a.table_h; }

constexpr int kEntryThreads = 256;
static int blocks_of(int max_pages) { return (max_pages - 1) / kEntryThreads + 1; }  // of a list
int64_t entry_workgroups(const ckv_lists *l) { return (int64_t)l->batch * l->n_kv_heads * blocks_of(l->max_pages); }

// ---------------------------------------------------------------------------------------------
// Lists that become copies
// ---------------------------------------------------------------------------------------------
struct ForkArgs {
  ListArgs to;
  const int32_t *from;  // strides as to.table
  const int32_t *parent, *length;
  int32_t *length_out;
  int batch, blocks;    // workgroups of a list
};

// A thread for an entry. What it names from now on is counted up, what it named down, in any order: the list that becomes a copy's source still names its
// pages, so none of them looks free between. One launch: 32 lists of 2048 entries 3.4 us; up and down by a launch each 6.7.
__global__ void __launch_bounds__(kEntryThreads) fork_kernel(ForkArgs a) {
  const int l = blockIdx.x / a.blocks, e = blockIdx.x % a.blocks * kEntryThreads + threadIdx.x, b = l / a.to.heads;
  const int parent = a.parent[b];
  const bool goes_on = (unsigned)parent < (unsigned)a.batch;
  if (a.length_out && blockIdx.x % a.blocks == 0 && l % a.to.heads == 0)
    for (int g = threadIdx.x; g < a.to.Hkv; g += kEntryThreads) a.length_out[b * a.to.Hkv + g] = goes_on ? a.length[parent * a.to.Hkv + g] : 0;
  if (e >= a.to.max_pages) return;
  int32_t *entry = list_of(a.to, l) + e;
  const int before = *entry;
  int now = goes_on ? a.from[parent * a.to.table_b + l % a.to.heads * a.to.table_h + e] : -1;
  if (!in_pool(a.to, now)) now = -1;
  if (before == now) return;
  *entry = now;
  if (now >= 0 && add_across(a.to.refs + now, 1) == 0) take_page(a.to, now);
  if (in_pool(a.to, before)) release_page(a.to, before);
}

hipError_t launch_fork(const ckv_lists *lists, const int32_t *table, const int32_t *parent, int32_t *table_out, int32_t *refs, uint32_t *taken,
                       const int32_t *length, int32_t *length_out, hipStream_t stream) {
  ForkArgs a;
  a.to = list_args(lists, table_out, refs, taken);
  a.from = table;
  a.parent = parent;
  a.length = length;
  a.length_out = length_out;
  a.batch = lists->batch;
  a.blocks = blocks_of(lists->max_pages);
  hipLaunchKernelGGL(fork_kernel, dim3((unsigned)a.to.lists * a.blocks), dim3(kEntryThreads), 0, stream, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Pages that are given back
// ---------------------------------------------------------------------------------------------
// A thread for an entry: a launch (64 lists of 563 entries 3.4 us; 32 of 2048, all pages released, 5.4 among a graph's kernels).
__global__ void __launch_bounds__(kEntryThreads) free_kernel(ListArgs a, const int32_t *keep, int blocks) {
  const int l = blockIdx.x / blocks, e = blockIdx.x % blocks * kEntryThreads + threadIdx.x;
  int rows = 0;
  if (keep) {
    const int32_t *mine = keep + l / a.heads * a.Hkv;
    if (a.heads > 1) rows = mine[l % a.heads];
    else
      for (int g = 0; g < a.Hkv; ++g) rows = max(rows, mine[g]);
  }
  const int stay = rows <= 0 ? 0 : ((rows - 1) >> a.shift) + 1;
  if (e < stay || e >= a.max_pages) return;
  int32_t *entry = list_of(a, l) + e;
  const int p = *entry;
  if (p != -1) *entry = -1;
  if (in_pool(a, p)) release_page(a, p);
}

hipError_t launch_free(const ckv_lists *lists, int32_t *table, const int32_t *keep, int32_t *refs, uint32_t *taken, hipStream_t stream) {
  const ListArgs a = list_args(lists, table, refs, taken);
  const int blocks = blocks_of(a.max_pages);
  hipLaunchKernelGGL(free_kernel, dim3((unsigned)a.lists * blocks), dim3(kEntryThreads), 0, stream, a, keep, blocks);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Pages for rows to come
// ---------------------------------------------------------------------------------------------
struct ReserveArgs {
  ListArgs to;
  const int32_t *first, *end;  // [batch][Hkv]
  int32_t *copy, *result;
  int n_copy;
};

constexpr int kReserveThreads = 1024, kReserveWaves = kReserveThreads / kWave;
constexpr int kFreeAhead = 2 * kReserveThreads;  // free pages found ahead: a round takes kReserveThreads at most

// One workgroup, its entries in rounds of a thread each, in their order. Entries whose page others name too count it down by one each; what is left of its
// count are the entries elsewhere. Where none are left, the last entry keeps the page: all write their number into the count, negative, and the
// smallest stays. Then what is needed is known, and either the counts become what they are to be, or what they were.
// A chain of dependent steps: rows, entries, counts, and with shared pages three more of the counts. What can be is asked for beside it (the bits of the
// first free pages), and a call of one round, which a step's is, keeps its entries in registers: 64 lists of four entries each, no
// shared page 5 us, 32 lists with one shared page each 7; with all steps for all entries, from memory each time, 15 to 17.
__global__ void __launch_bounds__(kReserveThreads) reserve_kernel(ReserveArgs a) {
  __shared__ int s_off[kReserveThreads], s_entry[kReserveThreads];  // of the lists: entries in front, the first entry
  __shared__ int s_sum[2][kReserveWaves];
  __shared__ int s_free[kFreeAhead];
  __shared__ int s_shared;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int turn = 0;

  // Sum over the threads in front; `total` of all.
  auto scan = [&](int x, int &total) CKV_INLINE {
    const int upto = wave_inclusive(x);
    int *sums = s_sum[turn ^= 1];  // those of the scan before may still be read
    if (lane == kWave - 1) sums[wave] = upto;
    __syncthreads();
    const int others = lane < kReserveWaves ? sums[lane] : 0, all = wave_inclusive(others);
    total = (int)lane_value((uint32_t)all, kWave - 1);
    return upto - x + (int)lane_value((uint32_t)(all - others), wave);
  };
  auto done = [&]() CKV_INLINE {  // what all threads have done to the counts is there
    wait_vm_at_most<0>();
    __syncthreads();
  };
  const int words = (a.to.n_pages - 1) / 32 + 1;
  auto free_bits = [&](int64_t w) CKV_INLINE {
    uint32_t bits = w < words ? ~a.to.taken[w] : 0u;
    if (w == words - 1 && a.to.n_pages % 32) bits &= (1u << a.to.n_pages % 32) - 1u;
    return bits;
  };

  // The ranges of the lists from l0 on: entries of them all; s_off and s_entry for find().
  auto ranges = [&](int l0) CKV_INLINE {
    const int l = l0 + tid;
    int from = INT32_MAX, upto = 0;  // rows
    if (l < a.to.lists) {
      const int heads = a.to.heads > 1 ? 1 : a.to.Hkv, at = l / a.to.heads * a.to.Hkv + l % a.to.heads;
#pragma unroll 8
      for (int g = 0; g < heads; ++g) {
        const int f = max(a.first[at + g], 0), e = a.end[at + g];
        from = min(from, e > f ? f : INT32_MAX);
        upto = max(upto, e > f ? e : 0);
      }
    }
    const int e0 = from >> a.to.shift, e1 = upto > 0 ? min(((upto - 1) >> a.to.shift) + 1, a.to.max_pages) : 0;
    int total;
    s_off[tid] = scan(max(e1 - e0, 0), total);
    s_entry[tid] = e0;
    __syncthreads();
    return total;
  };
  auto find = [&](int l0, int i) CKV_INLINE {  // entry i of these ranges
    int lo = 0, hi = min(a.to.lists - l0, kReserveThreads) - 1;  // the last list that begins at or in front of i
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (s_off[mid] <= i) lo = mid;
      else hi = mid - 1;
    }
    return list_of(a.to, l0 + lo) + s_entry[lo] + i - s_off[lo];
  };

  // The first free pages, and how many there are. They become taken a word at a time, by the thread that has found them, up to the number that is needed
  // (a page at a time, the bits of a round, which lie side by side, are an atomic operation each).
  int64_t page = 0;        // free pages in front of it have been found
  int have = 0, used = 0;  // of s_free
  int wanted = 0;          // pages that are not taken yet, of those that are needed
  auto take = [&](int64_t w, uint32_t bits, int some) CKV_INLINE {  // the first `some` of the word's pages
    if (some <= 0 || bits == 0) return;
    uint32_t rest = bits;
    for (int i = __popc(bits); i > some; --i) rest &= ~(0x80000000u >> __clz((int)rest));
    __scoped_atomic_fetch_or(a.to.taken + w, rest, __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE);
  };
  int place = 0;  // of the thread's first page
  auto more_free = [&](uint32_t bits) CKV_INLINE {  // of the words from page / 32 on, a thread each
    const int64_t w = (page >> 5) + tid;
    int found;
    place = have + scan(__popc(bits), found);
    int to = place;
    for (uint32_t rest = bits; rest && to < kFreeAhead; rest &= rest - 1) s_free[to++] = (int)(w * 32 + __builtin_ctz(rest));
    if (wanted > 0) {
      const int upto = min(kFreeAhead, have + wanted);
      take(w, bits, upto - place);
      wanted -= min(found, upto - have);
    }
    __syncthreads();
    const bool full = have + found >= kFreeAhead;
    page = full ? (int64_t)s_free[kFreeAhead - 1] + 1 : ((page >> 5) + kReserveThreads) * 32;
    have = full ? kFreeAhead : have + found;
    return found;
  };
  const uint32_t first_bits = free_bits(tid);
  for (int i = tid; i < 2 * a.n_copy; i += kReserveThreads) a.copy[i] = -1;
  if (tid == 0) s_shared = 0;
  const int lists_entries = ranges(0);
  int all_free = more_free(first_bits);
  if (words > kReserveThreads) {
    int rest = 0, sum;
    for (int64_t w = kReserveThreads + tid; w < words; w += kReserveThreads) rest += __popc(free_bits(w));
    scan(rest, sum);
    all_free += sum;
  }
  // What a round needs: gives x > 0 its page, x = 2 a pair too. All threads together.
  int pairs = 0;  // written
  auto give = [&](int32_t *entry, int was, int x) CKV_INLINE {
    int total;
    const int at = scan((x > 0) | (x == 2) << 16, total);
    const int asked = total & 0xffff;
    if (have - used < asked) {
      const int left = have - used;
      const int keep = tid < left ? s_free[used + tid] : 0;  // less than a round's
      __syncthreads();
      if (tid < left) s_free[tid] = keep;
      used = 0;
      have = left;
      while (have < asked && page < a.to.n_pages) {
        uint32_t bits = free_bits((page >> 5) + tid);
        if (tid == 0) bits &= ~0u << (page & 31);
        more_free(bits);
      }
    }
    if (x > 0 && used + (at & 0xffff) < have) {  // as many were counted, unless somebody else changes the bits meanwhile
      const int now = s_free[used + (at & 0xffff)];
      if (x == 2) {
        const int pair = pairs + (at >> 16);
        a.copy[2 * (size_t)pair] = was;
        a.copy[2 * (size_t)pair + 1] = now;
      }
      *entry = now;
      store_across(a.to.refs + now, 1);
    }
    used += asked;
    pairs += total >> 16;
  };
  auto result = [&](int need, int leave) CKV_INLINE {  // whether there is enough; the pages that have been found are taken then
    const int missing = max(max(need - all_free, leave - a.n_copy), 0);
    if (tid == 0) {
      a.result[0] = missing;
      a.result[1] = missing ? 0 : leave;
    }
    if (missing == 0) {
      take(tid, first_bits, min(need, kFreeAhead) - place);
      wanted = need - min(need, have);
    }
    return missing == 0;
  };
  auto shared = [&](int p) CKV_INLINE { return in_pool(a.to, p) && load_across(a.to.refs + p) > 1; };

  if (a.to.lists <= kReserveThreads && lists_entries <= kReserveThreads) {
    int32_t *entry = tid < lists_entries ? find(0, tid) : nullptr;
    const int p = entry ? *entry : -1;
    int x = entry && !in_pool(a.to, p) ? 1 : 0;  // what the entry needs: nothing, a page (1), a page and a copy of the one that it names (2)
    bool keeps = false;                          // a page that all others leave
    const bool is_shared = entry && shared(p);
    if (is_shared) s_shared = 1;
    __syncthreads();
    if (s_shared) {
      if (is_shared) add_across(a.to.refs + p, -1);
      done();
      if (is_shared && load_across(a.to.refs + p) <= 0) min_across(a.to.refs + p, -1 - tid);
      done();
      if (is_shared) keeps = load_across(a.to.refs + p) == -1 - tid;
      if (is_shared && !keeps) x = 2;
    }
    int total;
    scan((x > 0) | (x == 2) << 16, total);
    if (result(total & 0xffff, total >> 16)) {
      if (keeps) store_across(a.to.refs + p, 1);
      give(entry, p, x);
    } else if (s_shared) {
      if (keeps) store_across(a.to.refs + p, 0);
      done();
      if (is_shared) add_across(a.to.refs + p, 1);
    }
    return;
  }

  // Calls `visit(entry or null, its number)` for every entry of the ranges, all threads together.
  auto entries = [&](auto visit) CKV_INLINE {
    int number = 0;
    for (int l0 = 0; l0 < a.to.lists; l0 += kReserveThreads) {
      const int total = ranges(l0);
      for (int i0 = 0; i0 < total; i0 += kReserveThreads) {
        const int i = i0 + tid;
        visit(i < total ? find(l0, i) : nullptr, number + i);
      }
      number += total;
      __syncthreads();
    }
  };
  // Without shared pages, as for prompts to come, entries need a page or nothing.
  int need = 0, leave = 0, all_need, all_leave;
  bool any = false;
  entries([&](int32_t *entry, int) CKV_INLINE {
    need += entry && !in_pool(a.to, *entry);
    any |= entry && shared(*entry);
  });
  if (any) s_shared = 1;
  scan(need, all_need);
  if (!s_shared) {
    if (result(all_need, 0)) entries([&](int32_t *entry, int) CKV_INLINE { give(entry, -1, entry && !in_pool(a.to, *entry)); });
    return;
  }
  // Counts above one are those of shared pages until they are counted down; then those that entries number, negative, are. So all entries are counted
  // down here, and whoever keeps a page counts it up again.
  entries([&](int32_t *entry, int) CKV_INLINE {
    if (entry && in_pool(a.to, *entry)) add_across(a.to.refs + *entry, -1);
  });
  done();
  entries([&](int32_t *entry, int number) CKV_INLINE {
    if (entry && in_pool(a.to, *entry) && load_across(a.to.refs + *entry) <= 0) min_across(a.to.refs + *entry, -1 - number);
  });
  done();
  auto need_of = [&](const int32_t *entry, int number) CKV_INLINE {
    if (!entry) return 0;
    if (!in_pool(a.to, *entry)) return 1;
    return load_across(a.to.refs + *entry) == -1 - number ? 0 : 2;
  };
  need = 0;
  entries([&](int32_t *entry, int number) CKV_INLINE {
    const int x = need_of(entry, number);
    need += x > 0;
    leave += x == 2;
  });
  scan(need, all_need);
  scan(leave, all_leave);
  if (!result(all_need, all_leave)) {
    entries([&](int32_t *entry, int number) CKV_INLINE {
      if (entry && in_pool(a.to, *entry) && load_across(a.to.refs + *entry) == -1 - number) store_across(a.to.refs + *entry, 0);
    });
    done();
    entries([&](int32_t *entry, int) CKV_INLINE {
      if (entry && in_pool(a.to, *entry)) add_across(a.to.refs + *entry, 1);
    });
    return;
  }
  entries([&](int32_t *entry, int number) CKV_INLINE {
    const int x = need_of(entry, number), was = entry ? *entry : -1;
    if (entry && x == 0) store_across(a.to.refs + was, 1);
    give(entry, was, x);
  });
}

hipError_t launch_reserve(const ckv_lists *lists, int32_t *table, const int32_t *first, const int32_t *end, int32_t *refs, uint32_t *taken,
                          int32_t *copy, int n_copy, int32_t *result, hipStream_t stream) {
  const ReserveArgs a = {list_args(lists, table, refs, taken), first, end, copy, result, n_copy};
  hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(kReserveThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ckv
