// Pages of the cache (include/mars_cache.h): given out, shared, given back.  The only state is refs: a page is free exactly
// when its count is zero, so there is no list of free pages to keep in order, and who gets which page depends on nothing but the tables.
#pragma once

#include "kv_format.h"

namespace mars {
namespace kv {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;

// Workspace of a reserve: per request what it wants, then the pages found and the copies to make.
struct ReserveSpace {
  int32_t *shared;  // [B] page in which the request's first new token goes, if that page has tokens already; -1
  int32_t *wants;   // [B] pages it gets; the copy among them is bit 30
  int32_t *begin;   // [B] first of them among the found
  int32_t *found;   // [pages]
  int32_t *copy_src, *copy_dst;  // [B]
  int32_t *copies;  // [1]
};
constexpr int kCopyBit = 1 << 30;

// Sum of v over the threads in front of this one, and over all.
__device__ __forceinline__ int scan(int v, int* sh, int& total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int x = v;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();  // (sh may still be read from the scan before)
  if (lane == kWave - 1) sh[wave] = x;
  __syncthreads();
  int front = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    if (w < wave) front += sh[w];
    total += sh[w];
  }
  return front + x - v;
}

// One work-group: requests' wants, the lowest free pages, the tables.
// What bounds it: the latency of a few dependent loads and barriers, and of the way through refs to the free pages
// (4 096 of them per step).
__global__ void __launch_bounds__(kPlanThreads) reserve_kernel(Cache c, const int32_t* __restrict__ seqs, const int32_t* __restrict__ n_new,
                                                               int B, int N, int32_t* __restrict__ status, ReserveSpace ws) {
  __shared__ int sh[kPlanWaves];
  __shared__ int tile[kPlanThreads];
  const int tid = threadIdx.x, P = 1 << c.log_page;

  // what every request needs; the page its first new token goes to
  for (int b = tid; b < B; b += kPlanThreads) {
    const int s = sequence_of(c, seqs, b);
    int shared = -1, wants = 0, why = MARS_KV_OK;
    if (s < 0) {
      why = MARS_KV_BAD_SEQUENCE;
    } else {
      const int len = max(c.lens[s], 0), held = min(max(c.held[s], 0), c.width), n = n_new ? min(max(n_new[b], 0), N) : N;
      const long need = (static_cast<long>(len) + n + P - 1) >> c.log_page;
      if (need > c.width) {
        why = MARS_KV_TOO_LONG;
      } else {
        wants = max(static_cast<int>(need) - held, 0);
        const int at = len >> c.log_page;
        if ((len & (P - 1)) && n > 0 && at < held) shared = page_of(c, s, len);
      }
    }
    ws.shared[b] = shared;
    ws.wants[b] = wants;
    if (status) status[b] = why;
  }
  __syncthreads();

  // a page that others hold too is copied, unless this is the last of its holders and all of them are here
  for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    const int mine = b < B ? ws.shared[b] : -1;
    const int holders = mine >= 0 ? c.refs[mine] : 0;
    int here = 0, later = 0;
    if (__syncthreads_or(holders > 1)) {
      for (int t0 = 0; t0 < B; t0 += kPlanThreads) {
        __syncthreads();
        tile[tid] = t0 + tid < B ? ws.shared[t0 + tid] : -1;
        __syncthreads();
        if (holders > 1) {
          const int m = min(kPlanThreads, B - t0);
          for (int i = 0; i < m; ++i) {
            const bool same = tile[i] == mine;
            here += same;
            later += same && t0 + i > b;
          }
        }
      }
    }
    if (holders > 1 && (later > 0 || holders > here)) ws.wants[b] = (ws.wants[b] + 1) | kCopyBit;
  }
  __syncthreads();

  // in order of the requests
  long demand = 0;
  for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int total;
    const int want = b < B ? ws.wants[b] & ~kCopyBit : 0;
    const int before = scan(want, sh, total);
    if (b < B) ws.begin[b] = static_cast<int>(min(demand + before, 0x3FFFFFFFl));
    demand += total;
  }

  // the lowest free pages, as many as are wanted
  const int most = static_cast<int>(min(demand, static_cast<long>(c.pages)));
  int have = 0;
  for (int p0 = 0; p0 < c.pages && have < most; p0 += kPlanThreads * 4) {
    const int p = p0 + tid * 4;
    int free[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) free[i] = p + i < c.pages && c.refs[p + i] == 0;
    int total;
    int at = have + scan(free[0] + free[1] + free[2] + free[3], sh, total);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (free[i] && at < most) ws.found[at] = p + i;
      at += free[i];
    }
    have += total;
  }
  have = min(have, most);
  __syncthreads();

  // the tables: a wave per request.  (A request that does not get all it wants gets nothing; begin only grows, so those behind
  // it that want any get nothing either.)
  int copies = 0;  // those in front, the same in all threads
  for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    const int want = b < B ? ws.wants[b] : 0;
    const bool fits = b < B && ws.begin[b] + (want & ~kCopyBit) <= have;
    const bool copy = fits && (want & kCopyBit);
    int total;
    const int rank = copies + scan(copy, sh, total);
    if (copy) {
      ws.copy_src[rank] = ws.shared[b];
      ws.copy_dst[rank] = ws.found[ws.begin[b]];
    }
    if (b < B && !fits && (want & ~kCopyBit) && status) status[b] = MARS_KV_NO_PAGES;
    copies += total;
  }
  if (tid == 0) *ws.copies = copies;
  const int lane = tid % kWave;
  for (int b = tid / kWave; b < B; b += kPlanWaves) {
    const int want = ws.wants[b] & ~kCopyBit, begin = ws.begin[b];
    const bool copy = (ws.wants[b] & kCopyBit) != 0;
    if (want == 0 || begin + want > have) continue;
    const int s = sequence_of(c, seqs, b);
    if (s < 0) continue;
    const int held = min(max(c.held[s], 0), c.width), fresh = want - copy;
    int32_t* row = c.page_table + static_cast<size_t>(s) * c.width;
    if (copy && lane == 0) {
      const int page = ws.found[begin];
      atomicSub(&c.refs[ws.shared[b]], 1);
      c.refs[page] = 1;
      row[max(c.lens[s], 0) >> c.log_page] = page;
    }
    for (int i = lane; i < fresh; i += kWave) {
      const int page = ws.found[begin + copy + i];
      c.refs[page] = 1;
      row[held + i] = page;
    }
    if (lane == 0) c.held[s] = held + fresh;
  }
  // the last holder of a page keeps it only if the others got their copies (the counts are read past the first cache, where the
  // subtractions above were made)
  __syncthreads();
  for (int b = tid; status && b < B; b += kPlanThreads)
    if (ws.shared[b] >= 0 && !(ws.wants[b] & kCopyBit) && status[b] == MARS_KV_OK &&
        __hip_atomic_load(&c.refs[ws.shared[b]], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) > 1)
      status[b] = MARS_KV_NO_PAGES;
}

// A work-group per pair.
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

// A work-group per sequence.  (What it holds is taken out in one step, so that a sequence named twice gives its pages back once.)
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
// since an ancestor's number is smaller.  The parents lie in LDS; a tree is a few levels deep, a chain of N nodes N.
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
