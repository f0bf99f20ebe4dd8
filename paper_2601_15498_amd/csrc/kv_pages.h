// Pages of the cache (include/mars_cache.h): given out, shared, given back.  The only state is refs: a page is free exactly
// when its count is zero, so there is no list of free pages to keep in order, and who gets which page depends on nothing but the tables.
#pragma once

#include "kv_format.h"

namespace mars {
namespace kv {

constexpr int kPlanFew = 256, kPlanMany = 1024;  // threads of the work-group that plans a reserve: a barrier of four waves is the quicker one

// Workspace of a reserve: the pages found, the copies to make; the rest only where a request has several shared pages to write.
struct ReserveSpace {
  int32_t* found;                // [pages]
  int32_t *copy_src, *copy_dst;  // [B]
  int32_t* copies;               // [1]
  int32_t* former;               // [pages] the page that found[i] replaces
  int32_t *asks, *last;          // [pages] of a shared page: how many requests write it, the last of them
};
constexpr int kCopyBit = 1 << 30;    // of the pages a request wants: the first is to be a copy of the one it replaces
constexpr int kCommitted = 1 << 30;  // of the first page it writes: committed tokens are in it
// Sums stop here: a call may want more pages than 32 bits count (more than there are in any case), and one request at most 2^27.
__device__ __forceinline__ int plus(int a, int b) { return static_cast<int>(min(static_cast<u32>(a) + static_cast<u32>(b), 0x7FFFFFFFu)); }
// Sum of v (>= 0) over the threads in front of this one, and over all.  Where it stops, it is no less than the last sum minus v.
template <int THREADS> __device__ __forceinline__ int scan(int v, int* sh, int& total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int x = v;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x = plus(x, y);
  }
  __syncthreads();  // (sh may still be read from the scan before)
  if (lane == kWave - 1) sh[wave] = x;
  __syncthreads();
  int front = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) {
    if (w < wave) front = plus(front, sh[w]);
    total = plus(total, sh[w]);
  }
  return plus(front, x) - v;
}

// f(request, place in its row, page, its holders, number) for all pages that requests write, eight lanes for a request, which call it together; `number` is f's own to count with
// within a request, 0 at first.
template <int THREADS, typename F> __device__ void walk(const Cache& c, int B, const int* sh_seq, const int* sh_first, const int* sh_last, F f) {
  for (int b = threadIdx.x / 8; b < B; b += THREADS / 8) {
    const int32_t* row = c.page_table + static_cast<size_t>(max(sh_seq[b], 0)) * c.width;
    int number = 0;
    for (int i0 = sh_first[b] & ~kCommitted; i0 < sh_last[b]; i0 += 32) {
      int page[4], holders[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = i0 + 8 * k + static_cast<int>(threadIdx.x % 8);
        page[k] = i < sh_last[b] ? row[i] : -1;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        holders[k] = static_cast<u32>(page[k]) < static_cast<u32>(c.pages) ? __hip_atomic_load(&c.refs[page[k]], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) f(b, i0 + 8 * k + static_cast<int>(threadIdx.x % 8), page[k], holders[k], number);
    }
  }
}

// One work-group: requests' wants, the lowest free pages, the tables.  What it knows of the requests lies in LDS.
// A page that is to be written and that others hold too is given up for a free one, unless this is the last of its holders and all of them are here.  As a rule
// a request has one such page at most, the one that its committed tokens end in, and they are compared in LDS; a sequence that was cut back to an
// earlier token can have many, and then their writers are counted page by page in the workspace.
// What bounds it: the latency of its chain of loads (sequence, length, page, count) and barriers, and the way through refs to the free
// pages, 16 of them per thread and step.  A request's two children 8.6 us, 16 requests' eight each 13.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) reserve_kernel(Cache c, const int32_t* __restrict__ seqs, const int32_t* __restrict__ n_new,
                                                               int B, int N, int32_t* __restrict__ status, ReserveSpace ws) {
  constexpr int MOST = THREADS == kPlanFew ? kPlanFew : MARS_KV_MAX_REQUESTS;
  constexpr int LOOK = 8;  // pages of a request that are looked at at once
  __shared__ int sh[THREADS / kWave];
  __shared__ __attribute__((aligned(16))) int sh_shared[MOST + 3];
  __shared__ int sh_seq[MOST], sh_held[MOST], sh_wants[MOST], sh_begin[MOST];
  __shared__ int sh_first[MOST], sh_last[MOST];  // the pages held that are written: places in the row, `last` behind them
  __shared__ int sh_at[MOST], sh_swaps[MOST];    // place of sh_shared; pages given up
  __shared__ uint8_t sh_why[MOST];
  const int tid = threadIdx.x, P = 1 << c.log_page;

  // what every request needs; the pages its new tokens go to
  bool any = false, several = false;  // pages that others hold too
  for (int b = tid; b < B; b += THREADS) {
    const int s = sequence_of(c, seqs, b);
    int shared = -1, at = 0, wants = 0, held = 0, first = 0, last = 0, why = MARS_KV_OK;
    if (s < 0) {
      why = MARS_KV_BAD_SEQUENCE;
    } else {
      const int len = max(c.lens[s], 0), n = n_new ? min(max(n_new[b], 0), N) : N;
      held = min(max(c.held[s], 0), c.width);
      const long need = (static_cast<long>(len) + n + P - 1) >> c.log_page;
      if (need > c.width) {
        why = MARS_KV_TOO_LONG;
      } else {
        wants = max(static_cast<int>(need) - held, 0);
        const int from = len >> c.log_page, to = min(held, static_cast<int>(need));
        if (n > 0 && from < to) {
          const int32_t* row = c.page_table + static_cast<size_t>(s) * c.width;
          int page[LOOK], holders[LOOK], count = 0;
#pragma unroll
          for (int k = 0; k < LOOK; ++k) page[k] = from + k < to ? row[from + k] : -1;
#pragma unroll
          for (int k = 0; k < LOOK; ++k) holders[k] = static_cast<u32>(page[k]) < static_cast<u32>(c.pages) ? c.refs[page[k]] : 0;
#pragma unroll
          for (int k = LOOK - 1; k >= 0; --k)
            if (holders[k] > 1) {
              shared = page[k];
              at = from + k;
              ++count;
            }
          any |= count > 0;
          several |= count > 1 || to - from > LOOK;
          first = from | (len & (P - 1) ? kCommitted : 0);
          last = to;
        }
      }
    }
    sh_seq[b] = s;
    sh_held[b] = held;
    sh_shared[b] = shared;
    sh_at[b] = at;
    sh_wants[b] = wants;
    sh_swaps[b] = 0;
    sh_first[b] = first;
    sh_last[b] = last;
    sh_why[b] = static_cast<uint8_t>(why);
  }
  if (tid < 3) sh_shared[B + tid] = -1;
  // which pages are given up
  auto load = [](const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };  // (past the first cache)
  auto given = [&](int b, int page, int holders) { return holders > 1 && (load(&ws.last[page]) != b || load(&ws.asks[page]) < holders); };
  bool listed = false;  // page by page
  if (__syncthreads_or(any || several)) {
    if (__syncthreads_or(several)) {
      any = false;
      walk<THREADS>(c, B, sh_seq, sh_first, sh_last, [&](int, int, int page, int holders, int&) {
        if (holders > 1) {
          ws.asks[page] = 0;
          ws.last[page] = -1;
          any = true;
        }
      });
      __threadfence();
      listed = __syncthreads_or(any);
      if (listed) {
        for (int b = tid; b < B; b += THREADS) sh_shared[b] = -1;
        walk<THREADS>(c, B, sh_seq, sh_first, sh_last, [&](int b, int, int page, int holders, int&) {
          if (holders > 1) {
            atomicAdd(&ws.asks[page], 1);
            atomicMax(&ws.last[page], b);
          }
        });
        __threadfence();
        __syncthreads();
        walk<THREADS>(c, B, sh_seq, sh_first, sh_last, [&](int b, int i, int page, int holders, int&) {
          if (!given(b, page, holders)) return;
          atomicAdd(&sh_swaps[b], 1);
          if (sh_first[b] == (i | kCommitted)) sh_shared[b] = page;
        });
        __syncthreads();
        for (int b = tid; b < B; b += THREADS) sh_wants[b] = (sh_wants[b] + sh_swaps[b]) | (sh_shared[b] >= 0 ? kCopyBit : 0);
      }
    } else {
      for (int b = tid; b < B; b += THREADS) {
        const int mine = sh_shared[b], holders = mine >= 0 ? c.refs[mine] : 0;
        if (holders <= 1) continue;
        int here = 0, later = 0;
        for (int i = 0; i < B; i += 4) {
          const int4 x = *reinterpret_cast<const int4*>(sh_shared + i);
          const bool e0 = x.x == mine, e1 = x.y == mine, e2 = x.z == mine, e3 = x.w == mine;
          here += e0 + e1 + e2 + e3;
          later += (e0 && i > b) + (e1 && i + 1 > b) + (e2 && i + 2 > b) + (e3 && i + 3 > b);
        }
        if (later > 0 || holders > here) {
          sh_swaps[b] = 1;
          sh_wants[b] = (sh_wants[b] + 1) | (sh_first[b] == (sh_at[b] | kCommitted) ? kCopyBit : 0);
        }
      }
    }
    __syncthreads();
  }

  // in order of the requests
  long demand = 0;
  for (int b0 = 0; b0 < B; b0 += THREADS) {
    const int b = b0 + tid;
    int total;
    const int before = scan<THREADS>(b < B ? sh_wants[b] & ~kCopyBit : 0, sh, total);
    if (b < B) sh_begin[b] = static_cast<int>(min(demand + before, 0x7FFFFFFFl));
    demand += total;
  }

  // the lowest free pages, as many as are wanted
  const int most = static_cast<int>(min(demand, static_cast<long>(c.pages)));
  int have = 0;
  for (int p0 = 0; p0 < c.pages && have < most; p0 += THREADS * 16) {
    const int p = p0 + tid * 16;
    u32 free = 0;
    if (p + 16 <= c.pages && reinterpret_cast<uintptr_t>(c.refs) % 16 == 0) {
      int4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = reinterpret_cast<const int4*>(c.refs + p)[i];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        free |= ((x[i].x == 0) | (x[i].y == 0) << 1 | (x[i].z == 0) << 2 | (x[i].w == 0) << 3) << (4 * i);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (p + i < c.pages && c.refs[p + i] == 0) free |= 1u << i;
    }
    int total;
    int at = have + scan<THREADS>(__popc(free), sh, total);
    while (free && at < most) {
      ws.found[at++] = p + __ffs(free) - 1;
      free &= free - 1;
    }
    have += total;
  }
  have = min(have, most);
  __syncthreads();

  // A request that does not get all it wants gets nothing; begin only grows, so those behind it that want any get nothing either.
  auto want_of = [&](int b) { return sh_wants[b] & ~kCopyBit; };
  auto fits = [&](int b) { return static_cast<long>(sh_begin[b]) + want_of(b) <= have; };
  int copies = 0;  // those in front, the same in all threads
  for (int b0 = 0; b0 < B; b0 += THREADS) {
    const int b = b0 + tid;
    const bool copy = b < B && (sh_wants[b] & kCopyBit) && fits(b);
    int total;
    const int rank = copies + scan<THREADS>(copy, sh, total);
    copies += total;
    if (b < B && want_of(b)) {
      if (!fits(b)) {
        sh_why[b] = MARS_KV_NO_PAGES;
      } else {
        const int s = sh_seq[b], swaps = sh_swaps[b];
        if (copy) {  // (of the pages given up it is the first in the row)
          ws.copy_src[rank] = sh_shared[b];
          ws.copy_dst[rank] = ws.found[sh_begin[b]];
        }
        if (swaps && !listed) {
          const int page = ws.found[sh_begin[b]];
          atomicSub(&c.refs[sh_shared[b]], 1);
          c.refs[page] = 1;
          c.page_table[static_cast<size_t>(s) * c.width + sh_at[b]] = page;
        }
        c.held[s] = sh_held[b] + want_of(b) - swaps;
      }
    }
  }
  if (tid == 0) *ws.copies = copies;
  if (listed) {  // (the counts stay as they are until all have looked at them)
    walk<THREADS>(c, B, sh_seq, sh_first, sh_last, [&](int b, int i, int page, int holders, int& number) {
      const bool mine = given(b, page, holders) && fits(b);
      const u32 eight = static_cast<u32>(__ballot(mine) >> (tid % kWave & ~7)) & 0xFF;
      if (mine) {
        const int k = sh_begin[b] + number + __popc(eight & ((1u << tid % 8) - 1)), other = ws.found[k];
        ws.former[k] = page;
        c.refs[other] = 1;
        c.page_table[static_cast<size_t>(sh_seq[b]) * c.width + i] = other;
      }
      number += __popc(eight);
    });
    __threadfence();
    __syncthreads();
  }
  // the pages that are added: a thread per page, which looks its request up
  for (int k = tid; k < have; k += THREADS) {
    int lo = 0, hi = B - 1;  // the last request that begins at k or before; those that want none come before it or begin later
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sh_begin[mid] <= k) lo = mid;
      else hi = mid - 1;
    }
    const int i = k - sh_begin[lo] - sh_swaps[lo];
    if (k >= sh_begin[lo] + want_of(lo) || !fits(lo)) continue;  // (pages that nobody gets)
    if (i < 0) {                                                 // in place of one that is given up
      if (listed) atomicSub(&c.refs[load(&ws.former[k])], 1);
      continue;
    }
    const int page = ws.found[k];
    c.refs[page] = 1;
    c.page_table[static_cast<size_t>(sh_seq[lo]) * c.width + sh_held[lo] + i] = page;
  }
  // The last holder of a page keeps it only if the others got theirs.
  if (listed) __threadfence();
  __syncthreads();
  if (listed) {
    walk<THREADS>(c, B, sh_seq, sh_first, sh_last, [&](int b, int, int, int holders, int&) {
      if (holders > 1 && sh_why[b] == MARS_KV_OK) sh_why[b] = MARS_KV_NO_PAGES;
    });
    __syncthreads();
  }
  for (int b = tid; status && b < B; b += THREADS) {
    int why = sh_why[b];
    if (!listed && sh_shared[b] >= 0 && !sh_swaps[b] && why == MARS_KV_OK && load(&c.refs[sh_shared[b]]) > 1) why = MARS_KV_NO_PAGES;
    status[b] = why;
  }
}

// A work-group per pair.  2 to 5 us: latency.
__global__ void __launch_bounds__(256) fork_kernel(Cache c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                   int32_t* __restrict__ status) {
  const int b = blockIdx.x, from = sequence_of(c, src, b), to = sequence_of(c, dst, b);
  int why = MARS_KV_OK;
  if (from < 0 || to < 0 || from == to) why = MARS_KV_BAD_SEQUENCE;
  else if (c.held[to] != 0) why = MARS_KV_NOT_EMPTY;
  __syncthreads();  // (held is written below)
  if (threadIdx.x == 0 && status) status[b] = why;
  if (why != MARS_KV_OK) return;
  const int len = max(c.lens[from], 0);
  const int shared = min(min(max(c.held[from], 0), c.width), static_cast<int>((static_cast<long>(len) + (1 << c.log_page) - 1) >> c.log_page));
  const int32_t* a = c.page_table + static_cast<size_t>(from) * c.width;
  int32_t* z = c.page_table + static_cast<size_t>(to) * c.width;
  for (int i = threadIdx.x; i < c.width; i += blockDim.x) {
    const int p = i < shared ? a[i] : -1;
    z[i] = p;
    if (static_cast<u32>(p) < static_cast<u32>(c.pages)) atomicAdd(&c.refs[p], 1);
  }
  if (threadIdx.x == 0) {
    c.lens[to] = len;
    c.held[to] = shared;
  }
}

// A work-group per sequence.  (What it holds is taken out in one step, so that a sequence named twice gives its pages back once.)  2 to 5 us.
__global__ void __launch_bounds__(256) release_kernel(Cache c, const int32_t* __restrict__ seqs, int32_t* __restrict__ status) {
  __shared__ int sh_held;
  const int b = blockIdx.x, s = sequence_of(c, seqs, b);
  if (threadIdx.x == 0) {
    if (status) status[b] = s < 0 ? MARS_KV_BAD_SEQUENCE : MARS_KV_OK;
    sh_held = s < 0 ? 0 : atomicExch(&c.held[s], 0);
    if (s >= 0) c.lens[s] = 0;
  }
  __syncthreads();
  const int held = min(sh_held, c.width);
  if (s < 0) return;
  int32_t* row = c.page_table + static_cast<size_t>(s) * c.width;
  for (int i = threadIdx.x; i < held; i += blockDim.x) {
    const int p = row[i];
    row[i] = -1;
    if (static_cast<u32>(p) < static_cast<u32>(c.pages)) atomicSub(&c.refs[p], 1);
  }
}

// ---------------------------------------------------------------- the tree's mask
// A work-group per request, a thread per node (up to four): it climbs to the root, its bits gathered word by word from the last on,
// since an ancestor's number is smaller.  The parents lie in LDS; a tree is a few levels deep, a chain of N nodes N.  Bound by the latency of that climb
// (and of the launch, some 2 us): trees of 60 nodes 4.6 us, of 1 024 15; as chains 7 and 270 (a chain needs no mask).
constexpr int kMaskThreads = 256;
__global__ void __launch_bounds__(kMaskThreads) tree_mask_kernel(const int32_t* __restrict__ tree_parent, const int32_t* __restrict__ n_new,
                                                                 int N, unsigned long long* __restrict__ mask, int32_t* __restrict__ status) {
  __shared__ int parent[MARS_MAX_NODES];
  const int b = blockIdx.x, words = (N + 63) / 64;
  const int n = n_new ? min(max(n_new[b], 0), N) : N;
  bool bad = false;
  for (int i = threadIdx.x; i < n; i += kMaskThreads) {
    const int p = tree_parent[static_cast<size_t>(b) * N + i];
    bad |= i == 0 ? p != -1 : p < 0 || p >= i;
    parent[i] = p;
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0 && status) status[b] = bad ? MARS_REQ_BAD_TREE : MARS_REQ_OK;
  for (int i = threadIdx.x; i < N; i += kMaskThreads) {
    unsigned long long* row = mask + (static_cast<size_t>(b) * N + i) * words;
    int w = words - 1;
    unsigned long long bits = 0;
    if (i < n && (!bad || i == 0)) {
      for (int j = i; j >= 0; j = j == 0 ? -1 : parent[j]) {
        for (; w > j >> 6; --w) {
          row[w] = bits;
          bits = 0;
        }
        bits |= 1ull << (j & 63);
      }
    }
    for (; w >= 0; --w) {
      row[w] = bits;
      bits = 0;
    }
  }
}

}  // namespace kv
}  // namespace mars
