// Who does what of an attention over the cache: the arguments of its kernels, and the deal of the work between work-groups, which each of them
// works out for itself from the lengths (nothing about them is known on the host).
#pragma once

#include "kv_format.h"

namespace mars {
namespace kv {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTile = 32;             // keys per wave and step
constexpr int kUnit = kWaves * kTile; // keys of a unit of work: each wave fetches a tile of it

struct AttnArgs {
  Cache c;
  size_t layer_offset;
  const int32_t* seqs;
  const int32_t* n_new;
  const unsigned long long* mask;
  const void* q;
  long q_request, q_node, q_head;
  void* out;
  long out_request, out_node, out_head;
  float* lse;
  float* partial;
  float scale_log2;
  int B, N, q_heads, group, words;
  int nodes;    // of a block of rows
  u32 least_share;  // units that a work-group takes at least
  u32 join_cost;    // how many units more than its share it takes rather than have blocks cut
  bool whole;       // the deal gives out whole items in any case
};

// ---------------------------------------------------------------- the deal
// A request's items are (cache head, block of `nodes` nodes), its units those of its items.  Under a mask a block has all the request's keys.
// In a chain it has those up to its last node, and blocks are taken in pairs, the last with the first and so on, so that every pair has about
// the same number of units: `per`, which is rounded up (what is left over of it is idle).
struct Request {
  int n, len, blocks, pairs;  // pairs: of blocks, or blocks
  u32 per;                    // units of a pair, or of a block
  __device__ __forceinline__ Request() {}
  __device__ __forceinline__ Request(const AttnArgs& a, int b) {
    const int s = sequence_of(a.c, a.seqs, b);
    n = a.n_new ? min(max(a.n_new[b], 0), a.N) : a.N;
    len = 0;
    if (s >= 0) len = min(max(a.c.lens[s], 0), a.c.width << a.c.log_page);
    else n = 0;
    blocks = (n + a.nodes - 1) / a.nodes;
    const bool paired = !a.mask && blocks > 1;
    pairs = paired ? (blocks + 1) / 2 : blocks;
    per = paired ? (2u * len + static_cast<u32>(blocks + 1) * a.nodes + 2 * (kUnit - 1)) / kUnit : static_cast<u32>(len + n + kUnit - 1) / kUnit;
  }
  __device__ __forceinline__ u32 items(const AttnArgs& a) const { return static_cast<u32>(a.c.heads) * pairs; }
  // Keys that a block's rows see at most.
  __device__ __forceinline__ int keys(const AttnArgs& a, int block) const { return len + (a.mask ? n : min(n, (block + 1) * a.nodes)); }
  __device__ __forceinline__ u32 block_units(const AttnArgs& a, int block) const { return static_cast<u32>(keys(a, block) + kUnit - 1) / kUnit; }
};
// Over the wave's lanes, lane 0 first: inside each row of 16 by shifts, then the rows in front through scalar registers (a scan by exchanges
// through LDS took a microsecond of every launch).  A lane whose source falls outside its row gets 0.
__device__ __forceinline__ u32 wave_scan(u32 v) {
  v += dpp<0x111>(v);  // row_shr 1, 2, 4, 8
  v += dpp<0x112>(v);
  v += dpp<0x114>(v);
  v += dpp<0x118>(v);
  const u32 t0 = __builtin_amdgcn_readlane(v, 15), t1 = __builtin_amdgcn_readlane(v, 31), t2 = __builtin_amdgcn_readlane(v, 47);
  const u32 row = threadIdx.x % kWave / 16;
  return v + (row > 0 ? t0 : 0) + (row > 1 ? t1 : 0) + (row > 2 ? t2 : 0);
}
__device__ __forceinline__ u32 wave_sum(u32 v) { return __builtin_amdgcn_readlane(wave_scan(v), kWave - 1); }
__device__ __forceinline__ u32 wave_max(u32 v) {
  v = max(v, dpp<0x111>(v));
  v = max(v, dpp<0x112>(v));
  v = max(v, dpp<0x114>(v));
  v = max(v, dpp<0x118>(v));
  return max(max(static_cast<u32>(__builtin_amdgcn_readlane(v, 15)), static_cast<u32>(__builtin_amdgcn_readlane(v, 31))),
             max(static_cast<u32>(__builtin_amdgcn_readlane(v, 47)), static_cast<u32>(__builtin_amdgcn_readlane(v, 63))));
}
// What a work-group's share of the units comes to, and a place in the deal, kept by every wave for itself: 64 requests at a time, one per lane.
// Where no work-group gets much more by it (join_cost units), whole items are given out and none is cut: then an item counts as two, one for each
// of its blocks.
struct Deal {
  const AttnArgs& a;
  Request mine;       // of request first + lane
  int first;
  u32 front, before;  // units in front of the 64, in front of the lane's request
  u32 sum;            // of the 64
  u32 total, share;
  bool whole;
  __device__ __forceinline__ u32 units(const Request& r) const { return whole ? 2 * r.items(a) : r.items(a) * r.per; }
  __device__ __forceinline__ void place(u32 units_in_front) {
    front = units_in_front;
    const u32 v = first + static_cast<int>(threadIdx.x % kWave) < a.B ? units(mine) : 0;
    const u32 x = wave_scan(v);
    before = front + x - v;
    sum = __builtin_amdgcn_readlane(x, kWave - 1);
  }
  __device__ __forceinline__ void load(int b0) {
    first = b0;
    mine = Request(a, min(b0 + static_cast<int>(threadIdx.x % kWave), a.B - 1));
  }
  __device__ __forceinline__ Deal(const AttnArgs& args, u32 groups) : a(args) {
    u32 items = 0, most = 0;
    total = 0;
    whole = false;
    for (int b = a.B - 1 & ~(kWave - 1); b >= 0; b -= kWave) {  // (ends at the first 64)
      load(b);
      const bool in = b + static_cast<int>(threadIdx.x % kWave) < a.B;
      items += wave_sum(in ? mine.items(a) : 0);
      total += wave_sum(in ? mine.items(a) * mine.per : 0);
      most = max(most, wave_max(in && mine.items(a) ? mine.per : 0));
    }
    share = total ? max((total + groups - 1) / groups, a.least_share) : 0;
    const u32 each = (items + groups - 1) / groups;
    whole = a.whole || each * most <= share + a.join_cost;
    if (whole) {
      share = 2 * each;
      total = 2 * items;
    }
    place(0);
  }
  // The block that unit u (not before an earlier call's) belongs to.
  struct Place {
    int b, head, block;
    u32 begin, count;   // of the block in the deal; count = 0: idle
    u32 offset;         // of u in the block; of idle ones: how many there are from u on
    Request r;
  };
  __device__ __forceinline__ Place find(u32 u) {
    while (u >= front + sum) {  // (u < total: there are more)
      load(first + kWave);
      place(front + sum);
    }
    const unsigned long long at = __ballot(before <= u && first + static_cast<int>(threadIdx.x % kWave) < a.B);
    // the last that begins at u or before; those without units that begin there too come before it or not at all
    const int lane = 63 - __builtin_clzll(at);
    Place p;
    p.b = first + lane;
    p.r.n = __builtin_amdgcn_readlane(mine.n, lane);
    p.r.len = __builtin_amdgcn_readlane(mine.len, lane);
    p.r.blocks = __builtin_amdgcn_readlane(mine.blocks, lane);
    p.r.pairs = __builtin_amdgcn_readlane(mine.pairs, lane);
    p.r.per = __builtin_amdgcn_readlane(mine.per, lane);
    const u32 local = u - __builtin_amdgcn_readlane(before, lane), per = whole ? 2 : p.r.per;
    const u32 item = local / per, in = local % per;
    p.head = item / p.r.pairs;
    p.block = item % p.r.pairs;
    const bool paired = p.r.pairs != p.r.blocks;  // (one block alone is no pair)
    const int late = paired ? p.r.blocks - 1 - p.block : p.block;
    const u32 those = whole ? 1 : paired ? p.r.block_units(a, late) : per;
    p.offset = in;
    if (in < those) {
      p.block = late;
      p.count = those;
    } else {
      p.offset = in - those;
      p.count = late == p.block ? 0 : whole ? 1 : p.r.block_units(a, p.block);
      if (p.offset >= p.count) {
        p.count = 0;
        p.offset = per - in;
      }
    }
    p.begin = u - p.offset;
    return p;
  }
};

}  // namespace kv
}  // namespace mars
