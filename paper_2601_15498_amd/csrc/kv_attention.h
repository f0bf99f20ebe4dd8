// Attention of a step's nodes over the paged 4-bit cache (include/mars_cache.h):
//   o = sum_j p_j v_j / sum_j p_j,   p_j = exp2(c s_j - m),   s_j = q . k_j,   c = scale * log2(e),
// one pass over the keys with a running reference m and sum.
//
// A wave takes 16 RB query rows (nodes x query heads of one cache head) and tiles of 32 keys.  Both products run on
// v_mfma_f32_16x16x32_bf16 with the keys, then the values, as the first operand, straight from the packed codes in registers:
// no LDS and no barrier on the way, and the probabilities never leave the registers they are formed in.
//   scores    first operand: lane (r = l%16, g = l/16) holds row r of a block of 16 keys, a quarter (D/4) of its channels, which is
//             contiguous in the page, with one scale (D = 256: two).  The order of the channels inside the product is free, so the queries are loaded
//             to match.  Row 4g + i of block b is the tile's key 8g + 4b + i, so that a lane ends up with the scores of the eight
//             keys 8g .. 8g + 7 for its query, in order --
//   values    -- which is what the second product's second operand holds.  Its first one: lane (r, g) has eight keys 8g .. 8g + 7 of D/16
//             channels of its own, in the page contiguous as well (that is what the values' layout is for).  A conversion gives two
//             channels of one key, the product takes two keys of one channel: a byte permutation per two values in between.
// The conversions are exact (a code times a power of two is a bf16 value).
//
// Few rows: the four waves of a work-group take every fourth tile of the same rows and meet in LDS at the end (KEYS).  Many: each
// wave has rows of its own (ROWS).  The work -- all tiles of all (request, cache head, block of rows) items -- is dealt out evenly: a
// work-group takes a run of tiles that may begin and end inside an item; what it has of such an item goes to the workspace, and
// merge_kernel joins the pieces.  Every work-group works out the deal from the lengths by itself.
#pragma once

#include <type_traits>

#include "kv_format.h"
#include "kv_rows.h"

namespace mars {
namespace kv {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTile = 32;             // keys per wave and step
constexpr int kUnit = kWaves * kTile; // keys of a unit of work: each wave fetches a tile of it
constexpr float kFloor = -3.0e38f;    // the reference before the first key that counts
constexpr float kSlack = 8.0f;        // how far (in powers of two) scores may pass the reference before it is moved up

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
  bool whole;   // the deal gives out whole items
};

__device__ __forceinline__ float max3(float a, float b, float c) {  // (written out: fmaxf would first quiet each operand)
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ float over_groups_max(float v) {  // over the four lanes that share l % 16
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float over_groups_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
__device__ __forceinline__ bf16x8 as_bf16x8(u32 a, u32 b, u32 c, u32 d) { return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d}); }
__device__ __forceinline__ u32 round_pair(float a, float b) { return __builtin_bit_cast(u32, __builtin_convertvector(f32x2{a, b}, bf16x2)); }
__device__ __forceinline__ float low_half(u32 w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(u32 w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two fp32 numbers as TERMS bf16 each whose sum is the number (to 24 bits with three).
template <int TERMS> __device__ __forceinline__ void split_pair(float a, float b, u32 (&t)[TERMS]) {
#pragma unroll
  for (int k = 0; k < TERMS; ++k) {
    t[k] = round_pair(a, b);
    if (k + 1 < TERMS) {
      a -= low_half(t[k]);
      b -= high_half(t[k]);
    }
  }
}

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
// Where no work-group gets much more by it (kJoinCost), whole items are given out and none is cut: then an item counts as two, one for each
// of its blocks.
constexpr u32 kJoinCost = 8;  // units; two prompts of 2 048, every pair of blocks with a work-group of its own: 50 units instead of 45, and the
                              // pieces' 134 MB neither written nor read
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
    share = (total + groups - 1) / groups;
    const u32 each = (items + groups - 1) / groups;
    whole = a.whole || each * most <= share + kJoinCost;
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

// ---------------------------------------------------------------- tiles on their way through LDS
// A tile of 32 keys in LDS: codes of the keys, codes of the values, then the scales of both.  Sixteen bytes go from memory to LDS per lane and
// instruction, past the registers, to places that follow each other; which sixteen they are is chosen so that the reads below find
// sixteen lanes' pieces on sixteen different groups of four banks.
template <int D> struct Tile {
  static constexpr int kCodes = 16 * D, kScales = D <= 128 ? 256 : 512;  // bytes
  static constexpr int kBytes = 2 * kCodes + kScales;
  static constexpr int kCodeLoads = kCodes / 1024, kScaleLoads = kScales / 256;
  static constexpr int kLoads = 2 * kCodeLoads + kScaleLoads;
  static constexpr int S = D / 32, VW = D == 256 ? 16 : 8;
  // Where sixteen bytes of the keys' codes stand: piece p (of D/32) of token t.
  __device__ static __forceinline__ u32 key_slot(u32 t, u32 p) {
    if (D == 64) return (t ^ (t >> 1 & 4)) * 2 + (p ^ (t >> 4 & 1));
    if (D == 128) return t * 4 + (p ^ (t >> 3 & 3));
    return t * 8 + (p ^ (t >> 2 & 6) ^ (t >> 1 & 1));
  }
  // And which piece of which token stands at `slot`: offset in the page's codes (from the tile's first token on).
  __device__ static __forceinline__ u32 key_source(u32 slot) {
    if (D == 64) {
      const u32 row = slot >> 1, t = row ^ (row >> 1 & 4);
      return t * 32 + ((slot & 1) ^ (t >> 4 & 1)) * 16;
    }
    if (D == 128) {
      const u32 t = slot >> 2;
      return t * 64 + ((slot & 3) ^ (t >> 3 & 3)) * 16;
    }
    const u32 t = slot >> 3;
    return t * 128 + ((slot & 7) ^ (t >> 2 & 6) ^ (t >> 1 & 1)) * 16;
  }
  // The same for the values: half h of dword column c (its eight tokens) of octet o.
  __device__ static __forceinline__ u32 value_slot(u32 o, u32 c, u32 h) {
    if (D == 64) return (o * 8 + c) * 2 + h;
    if (D == 128) return (o * 16 + c) * 2 + (h ^ (c >> 3));
    return (o * 16 + (c >> 1)) * 4 + ((((c & 1) << 1) | h) ^ (c >> 3));
  }
  __device__ static __forceinline__ u32 value_source(u32 slot) {
    if (D == 64) return slot * 16;
    if (D == 128) return (slot ^ (slot >> 4 & 1)) * 16;
    return (slot ^ (slot >> 4 & 3)) * 16;
  }
};
__device__ __forceinline__ u32 lds_address(const void* p) {
  return static_cast<u32>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)p));
}
// To LDS from byte address `lds` on, lane after lane.  (Written by hand: behind the compiler's own form of these loads every read of
// LDS waits for all that is in flight.  The wait states: a scalar operand can come from a vector instruction just before.)
template <int BYTES> __device__ __forceinline__ void buffer_to_lds(__amdgpu_buffer_rsrc_t rows, u32 at, u32 base, u32 lds) {
  if constexpr (BYTES == 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(at), "s"(rows), "s"(base) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(lds), "v"(at), "s"(rows), "s"(base) : "memory", "m0");
}
template <int BYTES> __device__ __forceinline__ void global_to_lds(const uint8_t* at, u32 lds) {
  if constexpr (BYTES == 16) asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(at) : "memory", "m0");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(at) : "memory", "m0");
}
template <int LEFT> __device__ __forceinline__ void arrived() {  // all loads of this wave but the last LEFT
  static_assert(LEFT >= 0 && LEFT < 64, "the counter's range");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
}
constexpr int kBufferFlags = 0x00020000;  // untyped buffer, 32-bit data format

// Fetches a wave's tiles of one piece of work, unit after unit.  UNIFORM: pages of 32 tokens and more, so that a tile lies in one page (a
// buffer, which the loads cannot leave).  Otherwise an octet does.  The page numbers of the next units lie in one register, a lane each: a load of the
// compiler's own in every unit would be waited for together with all that is in flight.
template <int D, bool UNIFORM> struct Fetch {
  using X = Tile<D>;
  static constexpr int kSpan = UNIFORM ? kWave : kWave / 4;  // units whose pages are known at a time
  const AttnArgs& a;
  const int32_t* row;  // of the page table
  int head, end, t0;   // keys there are; the next tile's first
  int ids, at;         // pages, which of them is next
  __device__ __forceinline__ Fetch(const AttnArgs& a_, int s, int head_, int end_, int from)
      : a(a_), row(a_.c.page_table + static_cast<size_t>(s) * a_.c.width), head(head_), end(end_), t0(from) {
    look_up();
  }
  // (past the end: the last position's page; -1 past the table)
  __device__ __forceinline__ void look_up() {
    const int lane = threadIdx.x % kWave, t = UNIFORM ? t0 + lane * kUnit : t0 + lane / 4 * kUnit + lane % 4 * 8;
    const int i = min(t, end - 1) >> a.c.log_page;
    ids = i < a.c.width ? row[i] : -1;
    asm volatile("" : "+v"(ids));  // waited for here, and not wherever it is next read
    at = 0;
  }
  // Octet (of the tile's four) that a lane's share of load i of the codes, or of the scales, belongs to.
  __device__ static __forceinline__ int code_octet(int i) { return (i * kWave + static_cast<int>(threadIdx.x % kWave)) / (D / 4); }
  __device__ static __forceinline__ int scale_octet() {
    const int lane = threadIdx.x % kWave;
    return D == 256 ? lane / 16 : D == 128 ? lane % 32 / 8 : lane % 16 / 4;
  }
  // The next tile to LDS.  Returns which of its octets have no page (bit by bit).
  __device__ __forceinline__ u32 next(u32 lds) {
    if (at == kSpan) look_up();
    const u32 lane = threadIdx.x % kWave, lp = a.c.log_page, in_page = (1u << lp) - 1;
    u32 bad;
    if constexpr (UNIFORM) {
      const u32 id = __builtin_amdgcn_readlane(ids, at);
      bad = id >= static_cast<u32>(a.c.pages) ? 0xF : 0;
      const auto rows = __builtin_amdgcn_make_buffer_rsrc(head_of(a.c, a.layer_offset, bad ? 0 : id, head), 0, static_cast<int>(a.c.blk), kBufferFlags);
      const u32 t = static_cast<u32>(t0) & in_page, k0 = t * (D / 2), v0 = ((D / 2) << lp) + k0;
#pragma unroll
      for (int i = 0; i < X::kCodeLoads; ++i) buffer_to_lds<16>(rows, X::key_source(i * kWave + lane), k0, lds + i * 1024);
#pragma unroll
      for (int i = 0; i < X::kCodeLoads; ++i) buffer_to_lds<16>(rows, X::value_source(i * kWave + lane), v0, lds + X::kCodes + i * 1024);
      const u32 s0 = (D << lp) + t * (D / 32), of_values = (D / 32) << lp;
      if constexpr (D == 256) {
        buffer_to_lds<4>(rows, lane * 4, s0, lds + 2 * X::kCodes);
        buffer_to_lds<4>(rows, lane * 4, s0 + of_values, lds + 2 * X::kCodes + 256);
      } else {  // the keys' scales in lanes 0 .. 31 (D = 64: twice), the values' in the others
        buffer_to_lds<4>(rows, lane % (D / 4) * 4 + lane / 32 * of_values, s0, lds + 2 * X::kCodes);
      }
    } else {
      bad = __ballot(static_cast<u32>(ids) >= static_cast<u32>(a.c.pages)) >> (at * 4) & 0xF;
      const u32 last = static_cast<u32>(end - 1) & ~7u;  // (octets past the end: the last one's place)
      auto head_at = [&](int octet) {
        const int p = __shfl(ids, at * 4 + octet);
        return head_of(a.c, a.layer_offset, static_cast<u32>(p) < static_cast<u32>(a.c.pages) ? p : 0, head);
      };
#pragma unroll
      for (int i = 0; i < X::kCodeLoads; ++i) {
        const u32 o = code_octet(i), t = min(static_cast<u32>(t0) + 8 * o, last) & in_page;
        const uint8_t* at = head_at(o) + t * (D / 2) - o * (4 * D);
        global_to_lds<16>(at + X::key_source(i * kWave + lane), lds + i * 1024);
        global_to_lds<16>(at + ((D / 2) << lp) + X::value_source(i * kWave + lane), lds + X::kCodes + i * 1024);
      }
      const u32 o = scale_octet(), t = min(static_cast<u32>(t0) + 8 * o, last) & in_page;
      const uint8_t* scales = head_at(o) + (D << lp) + t * (D / 32) + lane % (D / 16) * 4;
      if constexpr (D == 256) {
        global_to_lds<4>(scales, lds + 2 * X::kCodes);
        global_to_lds<4>(scales + ((D / 32) << lp), lds + 2 * X::kCodes + 256);
      } else {
        global_to_lds<4>(scales + (lane >= 32 ? (D / 32) << lp : 0), lds + 2 * X::kCodes);
      }
    }
    t0 += kUnit;
    ++at;
    return bad;
  }
};
// What a lane has of a tile, in registers: sixteen keys' quarter twice, and eight keys' values.
template <int D> struct Keys {
  u32 k[2][D / 32], ks[2];
  __device__ __forceinline__ explicit Keys(const uint8_t* tile) {
    using X = Tile<D>;
    const u32 lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
    const uint8_t* scales = tile + 2 * X::kCodes;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const u32 t = (r >> 2) * 8 + 4 * b + (r & 3);
      if constexpr (D == 64) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(tile + X::key_slot(t, g >> 1) * 16 + (g & 1) * 8);
        k[b][0] = w[0]; k[b][1] = w[1];
        ks[b] = scales[t * 2 + (g >> 1)];
      } else {
#pragma unroll
        for (int h = 0; h < D / 128; ++h) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(tile + X::key_slot(t, 4 * h + g) * 16);
#pragma unroll
          for (int j = 0; j < 4; ++j) k[b][4 * h + j] = w[j];
        }
        if constexpr (D == 128) ks[b] = scales[t * 4 + g];
        else ks[b] = scales[t * 8 + g] | static_cast<u32>(scales[t * 8 + 4 + g]) << 8;
      }
    }
  }
};
// Two keys' values of the same channel beside each other: the low halves of two conversions, or the high ones.
__device__ __forceinline__ u32 low_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ u32 high_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

template <int D> struct Values {
  u32 v[Tile<D>::VW];
  u32x2 vs;
  __device__ __forceinline__ explicit Values(const uint8_t* tile) {
    using X = Tile<D>;
    const u32 lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
#pragma unroll
    for (int i = 0; i < X::VW / 4; ++i) {
      const u32 c = D == 64 ? r >> 1 : D == 128 ? r : 2 * r + (i >> 1);
      const u32x4 w = *reinterpret_cast<const u32x4*>(tile + X::kCodes + X::value_slot(g, c, i & 1) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * i + j] = w[j];
    }
    vs = *reinterpret_cast<const u32x2*>(tile + 2 * X::kCodes + (D <= 128 ? 128 : 256) + g * (D / 4) + (r * (D / 16)) / 32 * 8);
  }
  // Of the lane's eight keys only the first `there` count: past the end of the sequence memory holds anything, and 0 times that has to be 0.
  __device__ __forceinline__ void cut(int there) {
    vs[0] = there >= 4 ? vs[0] : there <= 0 ? 0 : vs[0] & ((1u << (8 * there)) - 1);
    vs[1] = there >= 8 ? vs[1] : there <= 4 ? 0 : vs[1] & ((1u << (8 * (there - 4))) - 1);
  }
  // f(n, fragment): operand n of the second product, channels c D/16 + n of lane column c, for all n.
  template <typename F> __device__ __forceinline__ void each(F f) const {
    const u32 scale[8] = {scale_at<0>(vs[0]), scale_at<1>(vs[0]), scale_at<2>(vs[0]), scale_at<3>(vs[0]),
                          scale_at<0>(vs[1]), scale_at<1>(vs[1]), scale_at<2>(vs[1]), scale_at<3>(vs[1])};
    auto pair = [&](auto byte, int n, const u32* words, u32 shift) {  // channels 2 byte, 2 byte + 1 of a dword column
      constexpr int BYTE = decltype(byte)::value;
      u32 y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = decode<BYTE>(words[j] >> shift, scale[j]);
      f(n, as_bf16x8(low_halves(y[0], y[1]), low_halves(y[2], y[3]), low_halves(y[4], y[5]), low_halves(y[6], y[7])));
      f(n + 1, as_bf16x8(high_halves(y[0], y[1]), high_halves(y[2], y[3]), high_halves(y[4], y[5]), high_halves(y[6], y[7])));
    };
    if constexpr (D == 64) {
      const u32 shift = (threadIdx.x & 1) * 16;
      pair(std::integral_constant<int, 0>{}, 0, v, shift);
      pair(std::integral_constant<int, 1>{}, 2, v, shift);
    } else {
#pragma unroll
      for (int h = 0; h < D / 128; ++h) {
        pair(std::integral_constant<int, 0>{}, 8 * h, v + 8 * h, 0);
        pair(std::integral_constant<int, 1>{}, 8 * h + 2, v + 8 * h, 0);
        pair(std::integral_constant<int, 2>{}, 8 * h + 4, v + 8 * h, 0);
        pair(std::integral_constant<int, 3>{}, 8 * h + 6, v + 8 * h, 0);
      }
    }
  }
};

// ---------------------------------------------------------------- a wave's rows
// The queries as the first product's second operand.  Three forms:
//   bf16 rows, D >= 128 (CODES): the keys' codes and scales go into the product as they are (4 bits by 8 bits, a scale per 32 channels), 128 channels at a time;
//     the queries go in as two 8-bit terms of four significant bits each, which is all that a bf16 number has, with one scale per row: what is lost of a
//     channel is below 2^-22 of the row's largest.  (The keys converted to bf16 instead: a third of the vector instructions that do not depend on the number of rows.)
//   bf16 rows, D = 64: keys converted to bf16, 32 channels at a time.
//   fp32 rows: the same with three bf16 terms.
typedef int i32x8 __attribute__((ext_vector_type(8)));
template <int D, typename T> constexpr bool kCodes = D >= 128 && !std::is_same<T, float>::value;

template <int D, int RB, typename T, bool CODES> struct Queries;
template <int D, int RB, typename T> struct Queries<D, RB, T, false> {
  static constexpr int S = D / 32, TERMS = std::is_same<T, float>::value ? 3 : 1;
  bf16x8 q[TERMS][RB][S];
  // Channels that lane group g takes in step s: eight from here on.
  __device__ static __forceinline__ int channel(int g, int s) { return D == 64 ? g * 16 + s * 8 : s / 4 * 128 + g * 32 + s % 4 * 8; }
  __device__ __forceinline__ void load(int rb, const T* row, bool live) {
    const int g = threadIdx.x % kWave / 16;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      u32 t[4][TERMS];
      const Eight e = load_eight(row + channel(g, s));
#pragma unroll
      for (int p = 0; p < 4; ++p) split_pair<TERMS>(live ? e.x[2 * p] : 0.0f, live ? e.x[2 * p + 1] : 0.0f, t[p]);
#pragma unroll
      for (int k = 0; k < TERMS; ++k) q[k][rb][s] = as_bf16x8(t[0][k], t[1][k], t[2][k], t[3][k]);
    }
  }
  __device__ __forceinline__ void scores(const Keys<D>& x, f32x4 (&sc)[2][RB]) const {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) sc[b][rb] = f32x4{0, 0, 0, 0};
      const u32 s0 = scale_at<0>(x.ks[b]), s1 = D == 256 ? scale_at<1>(x.ks[b]) : s0;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const u32 scale = s < 4 ? s0 : s1;
        const bf16x8 k = as_bf16x8(decode<0>(x.k[b][s], scale), decode<1>(x.k[b][s], scale), decode<2>(x.k[b][s], scale), decode<3>(x.k[b][s], scale));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int t = TERMS - 1; t >= 0; --t) sc[b][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[t][rb][s], sc[b][rb], 0, 0, 0);
      }
    }
  }
};
template <int D, int RB, typename T> struct Queries<D, RB, T, true> {
  static constexpr int H = D / 128;
  i32x8 q[2][RB][H];
  int scale[2][RB];  // of the row's two terms, as bytes like the keys'
  __device__ __forceinline__ void load(int rb, const T* row, bool live) {
    // The 8-bit operand's lane group g has channels 16 g .. + 15 and 64 + 16 g .. + 15 of each 128.
    const int g = threadIdx.x % kWave / 16;
    Eight e[H][4];
    u32 top = 0;
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        e[h][i] = load_eight(row + h * 128 + i / 2 * 64 + g * 16 + i % 2 * 8);
        top = max(top, top_bits(e[h][i]));
      }
    top = live ? top : 0;
    top = max(top, static_cast<u32>(__shfl_xor(static_cast<int>(top), 16)));
    top = max(top, static_cast<u32>(__shfl_xor(static_cast<int>(top), 32)));
    // The largest is 128 to 256 of the first term's steps; the second's are 32 times finer (what the first leaves is at most 8 of its own).
    const u32 exponent = max(top >> 23, 13u);
    const bool bad = top >= 0x7F800000u;  // a query that is not finite: its scores are NaN
    scale[0][rb] = bad ? 255 : static_cast<int>(exponent - 7);
    scale[1][rb] = bad ? 255 : static_cast<int>(exponent - 12);
    const float up = live ? __uint_as_float((261 - exponent) << 23) : 0.0f;  // 2^(7 - (exponent - 127))
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float x0 = e[h][i].x[4 * j] * up, x1 = e[h][i].x[4 * j + 1] * up, x2 = e[h][i].x[4 * j + 2] * up, x3 = e[h][i].x[4 * j + 3] * up;
          int first = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, 0, false);
          first = __builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, first, true);
          int second = __builtin_amdgcn_cvt_pk_fp8_f32((x0 - __builtin_amdgcn_cvt_f32_fp8(first, 0)) * 32.0f, (x1 - __builtin_amdgcn_cvt_f32_fp8(first, 1)) * 32.0f, 0, false);
          second = __builtin_amdgcn_cvt_pk_fp8_f32((x2 - __builtin_amdgcn_cvt_f32_fp8(first, 2)) * 32.0f, (x3 - __builtin_amdgcn_cvt_f32_fp8(first, 3)) * 32.0f, second, true);
          q[0][rb][h][2 * i + j] = first;
          q[1][rb][h][2 * i + j] = second;
        }
  }
  template <int H0> __device__ __forceinline__ f32x4 step(const Keys<D>& x, int b, int rb, f32x4 sc) const {
    const i32x8 k = {static_cast<int>(x.k[b][4 * H0]), static_cast<int>(x.k[b][4 * H0 + 1]), static_cast<int>(x.k[b][4 * H0 + 2]), static_cast<int>(x.k[b][4 * H0 + 3]), 0, 0, 0, 0};
    const int ks = static_cast<int>(x.ks[b]);
    sc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q[1][rb][H0], sc, 4, 0, H0, ks, 0, scale[1][rb]);  // (4: codes of 4 bits, 0: of 8)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q[0][rb][H0], sc, 4, 0, H0, ks, 0, scale[0][rb]);
  }
  __device__ __forceinline__ void scores(const Keys<D>& x, f32x4 (&sc)[2][RB]) const {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        sc[b][rb] = step<0>(x, b, rb, f32x4{0, 0, 0, 0});
        if constexpr (H == 2) sc[b][rb] = step<1>(x, b, rb, sc[b][rb]);
      }
  }
};

template <int D, int RB, typename T> struct Wave {
  static constexpr int NF = D / 16;             // blocks of 16 channels of the result
  static constexpr int TERMS = std::is_same<T, float>::value ? 3 : 1;
  Queries<D, RB, T, kCodes<D, T>> q;
  f32x4 o[NF][RB];
  float m[RB], l[RB];
  int node[RB];                                 // of this lane's rows; < 0: no row
  unsigned long long word[RB];                  // the row's mask, where it is one word

  // Rows row0 .. of the block of nodes from node0 on, which has `rows`.
  __device__ __forceinline__ void start(const AttnArgs& a, int b, int head, int node0, int row0, int rows) {
    const int r = threadIdx.x % 16;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int row = row0 + rb * 16 + r;
      const bool live = row < rows;
      const int in = live ? row / a.group : 0, h = live ? row - in * a.group : 0;
      node[rb] = live ? node0 + in : -1;
      word[rb] = a.mask && a.words == 1 ? a.mask[static_cast<size_t>(b) * a.N + node0 + in] : 0;
      q.load(rb, static_cast<const T*>(a.q) + b * a.q_request + static_cast<long>(node0 + in) * a.q_node + static_cast<long>(head * a.group + h) * a.q_head, live);
      m[rb] = kFloor;
      l[rb] = 0.0f;
#pragma unroll
      for (int f = 0; f < NF; ++f) o[f][rb] = f32x4{0, 0, 0, 0};
    }
  }
};

// Which of the keys first .. first + 7 (numbered from the first node on; committed ones are < 0) row `node` of n nodes sees.  `only`: its mask, if that
// is one word.
__device__ __forceinline__ u32 seen(const AttnArgs& a, unsigned long long only, int b, int node, int n, int first) {
  u32 bits;
  if (a.mask) {
    const unsigned long long* row = a.mask + (static_cast<size_t>(b) * a.N + node) * a.words;
    auto word = [&](int w) { return w < 0 ? ~0ull : w >= a.words ? 0ull : a.words == 1 ? only : row[w]; };
    const int w = first >> 6, shift = first & 63;
    bits = static_cast<u32>(word(w) >> shift);
    if (shift > 56) bits |= static_cast<u32>(word(w + 1) << (64 - shift));
  } else {
    const int k = node + 1 - first;
    bits = k >= 8 ? 0xFFu : k <= 0 ? 0u : (1u << k) - 1;
  }
  const int k = n - first;
  return bits & (k >= 8 ? 0xFFu : k <= 0 ? 0u : (1u << k) - 1);
}

// Probabilities of a tile's keys as the second product's second operand: TERMS bf16 terms each.
template <int D, int RB, typename T> struct Weights { u32 p[Wave<D, RB, T>::TERMS][RB][4]; };

// One tile.  `plain` (the same for the wave): every row sees all of it, and all of it is there.  Otherwise: request b has n nodes behind
// `len` tokens, the tile begins at t0; `poison`: the lane's octet has no page.
template <int D, int RB, typename T>
__device__ __forceinline__ void weigh(const AttnArgs& a, Wave<D, RB, T>& w, f32x4 (&sc)[2][RB], bool plain, int b, int len, int n, int t0, bool poison,
                                      Weights<D, RB, T>& y) {
  constexpr int NF = D / 16, TERMS = Wave<D, RB, T>::TERMS;
  const float c = a.scale_log2;
  __builtin_amdgcn_sched_barrier(0);  // (the values' conversions would be brought up to here, and their results kept)
  if (!plain) {
    const int first = t0 + static_cast<int>(threadIdx.x % kWave / 16) * 8 - len;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const u32 sees = w.node[rb] < 0 ? 0u : seen(a, w.word[rb], b, w.node[rb], n, first);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float s = poison ? __builtin_nanf("") : sc[k][rb][i];
          sc[k][rb][i] = sees >> (4 * k + i) & 1 ? s : -__builtin_inff();
        }
    }
  }
  float top[RB];
  bool up = false;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float t = max3(sc[0][rb][0], sc[0][rb][1], sc[0][rb][2]);
    t = max3(t, sc[0][rb][3], sc[1][rb][0]);
    t = max3(t, sc[1][rb][1], sc[1][rb][2]);
    t = max3(t, sc[1][rb][3], t);
    top[rb] = t * c;
    up |= top[rb] > w.m[rb] + kSlack;
  }
  if (__any(up)) {  // seldom after the first tiles
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float m = fmaxf(w.m[rb], over_groups_max(top[rb]));
      const float shrink = __builtin_amdgcn_exp2f(w.m[rb] - m);
      w.m[rb] = m;
      w.l[rb] *= shrink;
#pragma unroll
      for (int f = 0; f < NF; ++f) w.o[f][rb] *= shrink;
    }
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const float e0 = __builtin_amdgcn_exp2f(fmaf(sc[h / 2][rb][h % 2 * 2], c, -w.m[rb]));
      const float e1 = __builtin_amdgcn_exp2f(fmaf(sc[h / 2][rb][h % 2 * 2 + 1], c, -w.m[rb]));
      w.l[rb] += e0 + e1;
      u32 t[TERMS];
      split_pair<TERMS>(e0, e1, t);
#pragma unroll
      for (int k = 0; k < TERMS; ++k) y.p[k][rb][h] = t[k];
    }
  }
  __builtin_amdgcn_sched_barrier(0);
}
template <int D, int RB, typename T>
__device__ __forceinline__ void add_values(Wave<D, RB, T>& w, const Weights<D, RB, T>& y, int n, bf16x8 values) {
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int t = Wave<D, RB, T>::TERMS - 1; t >= 0; --t)
      w.o[n][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values, as_bf16x8(y.p[t][rb][0], y.p[t][rb][1], y.p[t][rb][2], y.p[t][rb][3]), w.o[n][rb], 0, 0, 0);
}

// Where the results of a lane go: element [f][i] of its row among the 16 from `row0` on is channel (4g + i) * D/16 + f0 + f.
template <int D, int F, typename T>
__device__ __forceinline__ void write_part(const AttnArgs& a, int b, int head, int node0, int row0, int rows, int f0, const f32x4 (&o)[F], float m, float l) {
  constexpr int C = D / 16;
  const int lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
  const int row = row0 + r;
  if (row >= rows) return;
  const int in = row / a.group, node = node0 + in, h = head * a.group + row - in * a.group;
  const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
  T* at = static_cast<T*>(a.out) + b * a.out_request + node * a.out_node + h * a.out_head + g * (4 * C) + f0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[F];
#pragma unroll
    for (int f = 0; f < F; ++f) x[f] = o[f][i] * inverse;
    if constexpr (std::is_same<T, float>::value) {
      if constexpr (F == 1) at[i * C] = x[0];
      else if constexpr (F == 2) *reinterpret_cast<f32x2*>(at + i * C) = f32x2{x[0], x[1]};
      else
#pragma unroll
        for (int f = 0; f < F; f += 4) *reinterpret_cast<f32x4*>(at + i * C + f) = f32x4{x[f], x[f + 1], x[f + 2], x[f + 3]};
    } else {
      if constexpr (F == 1) at[i * C] = static_cast<bf16_t>(round_pair(x[0], 0.0f));
      else if constexpr (F == 2) *reinterpret_cast<u32*>(at + i * C) = round_pair(x[0], x[1]);
      else if constexpr (F == 4) *reinterpret_cast<u32x2*>(at + i * C) = u32x2{round_pair(x[0], x[1]), round_pair(x[2], x[3])};
      else
#pragma unroll
        for (int f = 0; f < F; f += 8)
          *reinterpret_cast<u32x4*>(at + i * C + f) = u32x4{round_pair(x[f], x[f + 1]), round_pair(x[f + 2], x[f + 3]),
                                                            round_pair(x[f + 4], x[f + 5]), round_pair(x[f + 6], x[f + 7])};
    }
  }
  if (a.lse && g == 0 && f0 == 0)
    a.lse[(static_cast<size_t>(b) * a.N + node) * a.q_heads + h] =
        l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

// A piece in the workspace: [16 RB] references, [16 RB] sums, then the results lane by lane, [RB][D/16][64] of four.
template <int D, int RB> struct Piece {
  static constexpr int kFloats = 32 * RB + RB * (D / 16) * 256;
  float* at;
  __device__ __forceinline__ Piece(float* partial, long slot) : at(partial + slot * kFloats) {}
  __device__ __forceinline__ float& reference(int row) const { return at[row]; }
  __device__ __forceinline__ float& sum(int row) const { return at[16 * RB + row]; }
  __device__ __forceinline__ f32x4& part(int rb, int f, int lane) const {
    return reinterpret_cast<f32x4*>(at + 32 * RB)[(rb * (D / 16) + f) * kWave + lane];
  }
};

// Rows that see nothing because their request has fewer nodes (or no sequence): zeros.
template <typename T, int D> __device__ __forceinline__ void clear_rows(const AttnArgs& a, int b, int n) {
  const long items = static_cast<long>(a.N - n) * a.q_heads * (D / 8);
  for (long i = threadIdx.x; i < items; i += kThreads) {
    const int c = static_cast<int>(i % (D / 8)), h = static_cast<int>(i / (D / 8) % a.q_heads), node = n + static_cast<int>(i / (D / 8) / a.q_heads);
    T* at = static_cast<T*>(a.out) + b * a.out_request + node * a.out_node + h * a.out_head + c * 8;
    const u32 none[4] = {0, 0, 0, 0};
    store_eight(at, none);
    if (c == 0 && a.lse) a.lse[(static_cast<size_t>(b) * a.N + node) * a.q_heads + h] = -__builtin_inff();
  }
}

enum { KEYS = 0, ROWS = 1 };  // what the waves of a work-group divide between them
template <int MODE, int RB> constexpr int rows_per_block = MODE == KEYS ? 16 * RB : 64 * RB;
// Work-groups that have to fit a compute unit beside each other: what the compiler may give a wave of registers, and the ring of LDS.
constexpr int per_unit(int D, int RB, bool f32) { return D == 256 ? (RB == 1 && !f32 ? 2 : 1) : f32 ? 2 : RB == 1 ? 3 : 2; }
template <int D, int RB, typename T> constexpr int kPerUnit = per_unit(D, RB, std::is_same<T, float>::value);
constexpr int values_bytes(int D, int mode) { return mode == ROWS ? kWaves * (D / 16) * 1024 : 0; }  // of a unit's values as operands
constexpr int stages_of(int D, int mode, int groups) {  // units in the ring, the one that is worked on among them
  const int n = (160 * 1024 / groups - 1024 - values_bytes(D, mode)) / (kWaves * (32 * D + (D <= 128 ? 256 : 512)));
  return n > 4 ? 4 : n;
}

template <int D, int RB, typename T, int MODE, bool UNIFORM>
__global__ void __launch_bounds__(kThreads, (kPerUnit<D, RB, T>)) attention_kernel(AttnArgs a) {
  using X = Tile<D>;
  constexpr int NF = D / 16, STAGES = stages_of(D, MODE, kPerUnit<D, RB, T>);
  static_assert(STAGES >= 2, "a unit in flight while another is worked on");
  constexpr int kJoin = MODE == KEYS ? 2 * RB * NF * 1024 : 0;  // bytes for two waves' results
  constexpr int kRing = STAGES * kWaves * X::kBytes;
  __shared__ __attribute__((aligned(1024))) uint8_t sh_ring[kRing > kJoin ? kRing : kJoin];
  __shared__ __attribute__((aligned(16))) u32x4 sh_values[MODE == ROWS ? kWaves : 1][MODE == ROWS ? NF : 1][kWave];
  __shared__ u32 sh_bad[STAGES][kWaves];
  __shared__ float sh_m[MODE == KEYS ? 4 : 1][16 * RB], sh_l[MODE == KEYS ? 4 : 1][16 * RB];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;

  if (a.n_new || a.seqs)  // (otherwise every request has N nodes)
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
      const int n = Request(a, b).n;
      if (n < a.N) clear_rows<T, D>(a, b, n);
    }
  Deal deal(a, gridDim.x);
  const u32 share = deal.share;
  // neighbours in the deal on the same die (block index mod 8)
  const u32 per_die = gridDim.x >> 3;
  const u32 group = (blockIdx.x & 7) * per_die + (blockIdx.x >> 3);
  const unsigned long long my_begin = static_cast<unsigned long long>(group) * share;
  if (my_begin >= deal.total) return;
  const u32 unit0 = static_cast<u32>(my_begin), unit1 = static_cast<u32>(min(my_begin + share, static_cast<unsigned long long>(deal.total)));
  const u32 ring = lds_address(sh_ring);

  Wave<D, RB, T> w;
  for (u32 u = unit0; u < unit1;) {
    const auto p = deal.find(u);
    if (p.count == 0) {
      u += p.offset;
      continue;
    }
    const u32 taken = min(p.count - p.offset, unit1 - u);
    const bool whole = taken == p.count;
    const int units = static_cast<int>(deal.whole ? p.r.block_units(a, p.block) : taken);
    const int node0 = p.block * a.nodes, rows = min(a.nodes, p.r.n - node0) * a.group, row0 = MODE == ROWS ? wave * 16 * RB : 0;
    const int len = p.r.len, n = p.r.n, end = len + n;
    // no row of this wave sees keys from here on (-1: it has no rows)
    const int limit = row0 >= rows ? 0 : a.mask ? end : len + 1 + node0 + (min(rows, row0 + 16 * RB) - 1) / a.group;
    const int from = static_cast<int>(p.offset) * kUnit;
    // (in front of the queries' loads; LDS is free: the piece before ended with a barrier)
    Fetch<D, UNIFORM> fetch(a, sequence_of(a.c, a.seqs, p.b), p.head, end, from + wave * kTile);
    u32 stage = 0;
    auto issue = [&](u32 to) {
      const u32 bad = fetch.next(ring + (to * kWaves + wave) * X::kBytes);
      if (lane == 0) sh_bad[to][wave] = bad;
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
      if (i < units) issue(i);
    w.start(a, p.b, p.head, node0, row0, rows);

    for (int unit = 0; unit < units; ++unit) {
      // this wave's tile of the unit is there; with a barrier, all are, and nobody reads the unit before any more
      if (unit + STAGES - 1 <= units) arrived<(STAGES - 2) * X::kLoads>();
      else arrived<0>();
      if (MODE == ROWS) __builtin_amdgcn_s_barrier();
      if (unit + STAGES - 1 < units) issue(stage == 0 ? STAGES - 1 : stage - 1);
      const int t_unit = from + unit * kUnit;
      if constexpr (MODE == KEYS) {
        const int t0 = t_unit + wave * kTile;
        if (t0 < limit) {
          const uint8_t* tile = sh_ring + (stage * kWaves + wave) * X::kBytes;
          const u32 bad = __builtin_amdgcn_readfirstlane(sh_bad[stage][wave]);
          const bool plain = t0 + kTile <= len && bad == 0, poison = bad >> g & 1;
          const Keys<D> keys(tile);
          Values<D> values(tile);
          f32x4 sc[2][RB];
          w.q.scores(keys, sc);
          Weights<D, RB, T> y;
          weigh<D, RB, T>(a, w, sc, plain, p.b, len, n, t0, poison, y);
          if (!plain) values.cut(poison ? 0 : end - t0 - 8 * g);
          values.each([&](int f, bf16x8 v) { add_values<D, RB, T>(w, y, f, v); });
        }
      } else {
        // A tile's scores are under way on the matrix cores while the one before it is weighed, the first one's while each wave
        // converts the values of its tile for all.
        const uint8_t* const tiles = sh_ring + stage * kWaves * X::kBytes;
        f32x4 sc[2][2][RB];
        w.q.scores(Keys<D>(tiles), sc[0]);
        {
          const int t0 = t_unit + wave * kTile;
          const u32 bad = __builtin_amdgcn_readfirstlane(sh_bad[stage][wave]);
          Values<D> values(sh_ring + (stage * kWaves + wave) * X::kBytes);
          if (t0 + kTile > end || bad) values.cut(bad >> g & 1 ? 0 : end - t0 - 8 * g);
          values.each([&](int f, bf16x8 v) { sh_values[wave][f][lane] = __builtin_bit_cast(u32x4, v); });
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // (what is in flight from memory stays so)
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
          const int t0 = t_unit + i * kTile;
          if (t0 >= limit) break;
          const u32 bad = __builtin_amdgcn_readfirstlane(sh_bad[stage][i]);
          u32x4 v[NF];
#pragma unroll
          for (int f = 0; f < NF; ++f) v[f] = sh_values[i][f][lane];
          if (i + 1 < kWaves) w.q.scores(Keys<D>(tiles + (i + 1) * X::kBytes), sc[(i + 1) % 2]);
          Weights<D, RB, T> y;
          weigh<D, RB, T>(a, w, sc[i % 2], t0 + kTile <= len && bad == 0, p.b, len, n, t0, bad >> g & 1, y);
#pragma unroll
          for (int f = 0; f < NF; ++f) add_values<D, RB, T>(w, y, f, __builtin_bit_cast(bf16x8, v[f]));
        }
      }
      stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) w.l[rb] = over_groups_sum(w.l[rb]);
    __syncthreads();  // the ring is free

    if (MODE == KEYS) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        if (lane < 16) {
          sh_m[wave][rb * 16 + r] = w.m[rb];
          sh_l[wave][rb * 16 + r] = w.l[rb];
        }
      __syncthreads();
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        float m = kFloor, l = 0.0f;
#pragma unroll
        for (int v = 0; v < 4; ++v) m = fmaxf(m, sh_m[v][rb * 16 + r]);
#pragma unroll
        for (int v = 0; v < 4; ++v) l += sh_l[v][rb * 16 + r] * __builtin_amdgcn_exp2f(sh_m[v][rb * 16 + r] - m);
        const float shrink = __builtin_amdgcn_exp2f(w.m[rb] - m);
#pragma unroll
        for (int f = 0; f < NF; ++f) w.o[f][rb] *= shrink;
        w.m[rb] = m;
        w.l[rb] = l;
      }
      // waves 2 and 3 to 0 and 1, then 1 to 0
#pragma unroll
      for (int half = 2; half >= 1; half >>= 1) {
        f32x4* const sh = reinterpret_cast<f32x4*>(sh_ring) + (wave & (half - 1)) * (RB * NF * kWave) + lane;
        if (wave >= half && wave < 2 * half) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int f = 0; f < NF; ++f) sh[(rb * NF + f) * kWave] = w.o[f][rb];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int f = 0; f < NF; ++f) w.o[f][rb] += sh[(rb * NF + f) * kWave];
        }
        __syncthreads();
      }
    }
    if (MODE == ROWS || wave == 0) {
      if (whole) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          f32x4 o[NF];
#pragma unroll
          for (int f = 0; f < NF; ++f) o[f] = w.o[f][rb];
          write_part<D, NF, T>(a, p.b, p.head, node0, row0 + rb * 16, rows, 0, o, w.m[rb], w.l[rb]);
        }
      } else {
        // the first piece of the group's run, or its last one
        const long slot = (static_cast<long>(group) * 2 + (u == unit0 ? 0 : 1)) * (MODE == ROWS ? 4 : 1) + (MODE == ROWS ? wave : 0);
        const Piece<D, RB> piece(a.partial, slot);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          if (lane < 16) {
            piece.reference(rb * 16 + r) = w.m[rb];
            piece.sum(rb * 16 + r) = w.l[rb];
          }
#pragma unroll
          for (int f = 0; f < NF; ++f) piece.part(rb, f, lane) = w.o[f][rb];
        }
      }
    }
    u += taken;
  }
}

// Joins the pieces of blocks that were dealt to several work-groups: one work-group for every place where the deal cuts one, of which the
// first of a block takes it; a wave per 16 rows and quarter of the result's channels, eight pieces at a time under way (it is the latency of
// these loads that counts: a piece at a time took 8 us where this takes 4).
template <int D, int RB, typename T, int MODE>
__global__ void __launch_bounds__(kThreads) merge_kernel(AttnArgs a, u32 groups) {
  constexpr int NF = D / 16, F = NF / 4, AT_ONCE = D == 256 ? 4 : 8;
  Deal deal(a, groups);
  if (deal.whole) return;
  const u32 share = deal.share;
  const u32 cut = blockIdx.x + 1;
  const unsigned long long at = static_cast<unsigned long long>(cut) * share;
  if (at >= deal.total) return;
  const auto p = deal.find(static_cast<u32>(at));
  if (p.count == 0 || p.begin == at) return;          // cut between two blocks
  const u32 first = p.begin / share, last = (p.begin + p.count - 1) / share;
  if (cut != first + 1) return;                       // an earlier cut's
  const int node0 = p.block * a.nodes, rows = min(a.nodes, p.r.n - node0) * a.group;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane % 16;
  const int f0 = wave * F;
  constexpr int STRIPS = MODE == ROWS ? 4 * RB : RB;  // of 16 rows
  for (int strip = blockIdx.y; strip < STRIPS; strip += gridDim.y) {
  const int part = MODE == ROWS ? strip / RB : 0, rb = MODE == ROWS ? strip % RB : strip;
  if (strip * 16 >= rows) break;
  float m = kFloor, l = 0.0f;
  f32x4 o[F];
#pragma unroll
  for (int f = 0; f < F; ++f) o[f] = f32x4{0, 0, 0, 0};
  for (u32 x0 = first; x0 <= last; x0 += AT_ONCE) {
    float pm[AT_ONCE], pl[AT_ONCE];
    f32x4 po[AT_ONCE][F];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const u32 x = min(x0 + i, last);
      const u32 second = static_cast<unsigned long long>(x) * share >= p.begin ? 0 : 1;
      const Piece<D, RB> piece(a.partial, (static_cast<long>(x) * 2 + second) * (MODE == ROWS ? 4 : 1) + part);
      pm[i] = piece.reference(rb * 16 + r);
      pl[i] = piece.sum(rb * 16 + r);
#pragma unroll
      for (int f = 0; f < F; ++f) po[i][f] = piece.part(rb, f0 + f, lane);
    }
    const float before = m;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) m = fmaxf(m, pm[i]);
    const float shrink = __builtin_amdgcn_exp2f(before - m);
    l *= shrink;
#pragma unroll
    for (int f = 0; f < F; ++f) o[f] *= shrink;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if (x0 + i <= last) {
        const float weight = __builtin_amdgcn_exp2f(pm[i] - m);
        l += pl[i] * weight;
#pragma unroll
        for (int f = 0; f < F; ++f) o[f] += po[i][f] * weight;
      }
    }
  }
  write_part<D, F, T>(a, p.b, p.head, node0, strip * 16, rows, f0, o, m, l);
  }
}

}  // namespace kv
}  // namespace mars
