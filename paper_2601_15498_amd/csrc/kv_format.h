// The 4-bit cache's format on the device (include/mars_cache.h): where a token's bytes lie in a page, and the way from values to
// codes and back.  This file and those that include it are compiled with NaNs honoured.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/mars_cache.h"

namespace mars {
namespace kv {

constexpr int kWave = 64;
typedef unsigned int u32;
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
using bf16_t = uint16_t;

constexpr u32 kNanScale = 255;     // of all blocks of a key that (or whose value) is not finite
constexpr u32 kLeastScale = 1, kMostScale = 252;  // 6 * 2^(252 - 127) is finite; 2^(1 - 127) is no denormal

// Bytes of a head in a page of P = 2^log_page tokens.
__host__ __device__ __forceinline__ size_t head_bytes(int dim, int page) { return static_cast<size_t>(page) * (dim + dim / 16); }

// What a call knows of the cache: the pages of one layer (or of the first), the tables.
struct Cache {
  uint8_t* pool;
  int32_t *page_table, *lens, *held, *refs;
  size_t layer_bytes;  // of all pages of a layer
  u32 page_bytes, blk; // of a page in a layer; of a head in it
  int layers, pages, heads, log_page, sequences, width;
};

// Byte offsets within a head's part of a page.  t: token in the page.
template <int D> struct Place {
  __device__ static __forceinline__ u32 key(u32 t) { return t * (D / 2); }
  __device__ static __forceinline__ u32 value(u32 log_page, u32 t) { return ((D / 2) << log_page) + (t >> 3) * (D * 4) + (t & 7) * 4; }  // dword column c: + 32 c
  __device__ static __forceinline__ u32 key_scale(u32 log_page, u32 t) { return (D << log_page) + t * (D / 32); }
  __device__ static __forceinline__ u32 value_scale(u32 log_page, u32 t) {  // block s: + 8 s
    return (D << log_page) + ((D / 32) << log_page) + (t >> 3) * (D / 4) + (t & 7);
  }
};

// Sequence of request b, or -1.
__device__ __forceinline__ int sequence_of(const Cache& c, const int32_t* seqs, int b) {
  const int s = seqs ? seqs[b] : b;
  return static_cast<u32>(s) < static_cast<u32>(c.sequences) ? s : -1;
}
// Page that holds a sequence's tokens number position .., or -1.
__device__ __forceinline__ int page_of(const Cache& c, int s, int position) {
  const int i = position >> c.log_page;
  if (position < 0 || i >= c.width) return -1;
  const int p = c.page_table[static_cast<size_t>(s) * c.width + i];
  return static_cast<u32>(p) < static_cast<u32>(c.pages) ? p : -1;
}
__device__ __forceinline__ uint8_t* head_of(const Cache& c, size_t layer_offset, int page, int head) {
  return c.pool + layer_offset + static_cast<size_t>(page) * c.page_bytes + static_cast<size_t>(head) * c.blk;
}

// Eight channels of a row: as they lie in memory, and widened.
struct Eight { float x[8]; };
template <typename T> struct Raw;
template <> struct Raw<float> { f32x4 a, b; };
template <> struct Raw<bf16_t> { u32x4 a; };
__device__ __forceinline__ Raw<float> load_raw(const float* p) { return {*reinterpret_cast<const f32x4*>(p), *reinterpret_cast<const f32x4*>(p + 4)}; }
__device__ __forceinline__ Raw<bf16_t> load_raw(const bf16_t* p) { return {*reinterpret_cast<const u32x4*>(p)}; }
__device__ __forceinline__ Eight widen(const Raw<float>& r) { return {{r.a[0], r.a[1], r.a[2], r.a[3], r.b[0], r.b[1], r.b[2], r.b[3]}}; }
__device__ __forceinline__ Eight widen(const Raw<bf16_t>& r) {
  Eight e;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    e.x[2 * i] = __uint_as_float(r.a[i] << 16);
    e.x[2 * i + 1] = __uint_as_float(r.a[i] & 0xFFFF0000u);
  }
  return e;
}
template <typename T> __device__ __forceinline__ Eight load_eight(const T* p) { return widen(load_raw(p)); }
// Largest magnitude's bits; with a NaN or an infinity among them 0x7F800000 or more.
__device__ __forceinline__ u32 top_bits(const Eight& e) {
  u32 m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(e.x[i]) & 0x7FFFFFFFu);
  return m;
}
// The same over the four lanes that hold a block of 32 channels.
template <int CTRL> __device__ __forceinline__ u32 dpp(u32 v) {
  return static_cast<u32>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ u32 block_top(u32 m) {
  m = max(m, dpp<0xB1>(m));    // quad_perm [1,0,3,2]
  return max(m, dpp<0x4E>(m)); // quad_perm [2,3,0,1]
}
// Least exponent at which the largest magnitude is below 7 scales: floor(log2 m) - 2, one more from 1.75 * 2^k on.
__device__ __forceinline__ u32 scale_byte(u32 top) {
  const int e = static_cast<int>((top + 0x200000u) >> 23) - 2;
  return static_cast<u32>(min(max(e, static_cast<int>(kLeastScale)), static_cast<int>(kMostScale)));
}
// Eight codes.  The division by the scale is an exact product; the conversion rounds to nearest even and stops at 6.
__device__ __forceinline__ u32 encode(const Eight& e, u32 byte) {
  const float inverse = __uint_as_float((254u - byte) << 23);
  u32 w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[0] * inverse, e.x[1] * inverse, 1.0f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[2] * inverse, e.x[3] * inverse, 1.0f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[4] * inverse, e.x[5] * inverse, 1.0f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[6] * inverse, e.x[7] * inverse, 1.0f, 3);
  return w;
}
// Two codes (byte BYTE of w) as bf16, exactly.  Of the scale only bits 23 .. 30 count -- a byte of scales is
// brought there by one shift, whatever it leaves in the others -- and 255 gives NaN.
template <int BYTE> __device__ __forceinline__ u32 decode(u32 w, u32 scale) {
  return __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, __uint_as_float(scale), BYTE));
}
template <int BYTE> __device__ __forceinline__ u32 scale_at(u32 bytes) {
  static_assert(BYTE >= 0 && BYTE < 4, "");
  return BYTE == 3 ? bytes >> 1 : bytes << (23 - 8 * BYTE);
}

}  // namespace kv
}  // namespace mars
