// Tiles of the cache on their way from memory through a ring in LDS.
#pragma once

#include "kv_deal.h"

namespace mars {
namespace kv {

// A tile of 32 keys in LDS: codes of the keys, codes of the values, then the scales of both.  Sixteen bytes go from memory to LDS per lane and
// instruction, past the registers, to places that follow each other; which sixteen they are is chosen so that sixteen lanes' pieces are found on sixteen
// different groups of four banks, both by waves of 16 rows (which read tokens 8 i + j, i, j < 4, and those 4 on) and by those of 32 (16 tokens in a row).
template <int D> struct Tile {
  static constexpr int kCodes = 16 * D, kScales = D <= 128 ? 256 : 512;  // bytes
  static constexpr int kBytes = 2 * kCodes + kScales;
  static constexpr int kCodeLoads = kCodes / 1024, kScaleLoads = kScales / 256;
  static constexpr int kLoads = 2 * kCodeLoads + kScaleLoads;
  static constexpr int S = D / 32, VW = D == 256 ? 16 : 8;
  // Where sixteen bytes of the keys' codes stand: piece p (of D/32) of token t.
  __device__ static __forceinline__ u32 key_slot(u32 t, u32 p) {
    if (D == 64) return (t ^ (t >> 1 & 4)) * 2 + (p ^ turn(t));
    return t * (D / 32) + (p ^ turn(t));
  }
  __device__ static __forceinline__ u32 turn(u32 t) {
    if (D == 64) return (t >> 3 ^ t >> 4) & 1;
    if (D == 128) return (t >> 2 & 2) | ((t >> 2 ^ t >> 4) & 1);
    return (t << 1 & 4) | (t >> 2 & 2) | ((t >> 2 ^ t >> 4) & 1);
  }
  // And which piece of which token stands at `slot`: offset in the page's codes (from the tile's first token on).
  __device__ static __forceinline__ u32 key_source(u32 slot) {
    if (D == 64) {
      const u32 row = slot >> 1, t = row ^ (row >> 1 & 4);
      return t * 32 + ((slot & 1) ^ turn(t)) * 16;
    }
    const u32 t = slot / (D / 32);
    return t * (D / 2) + (slot % (D / 32) ^ turn(t)) * 16;
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
}  // namespace kv
}  // namespace mars
