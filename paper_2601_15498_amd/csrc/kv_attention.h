// Attention of a step's nodes over the paged 4-bit cache (include/mars_cache.h):
//   o = sum_j p_j v_j / sum_j p_j,   p_j = exp2(c s_j - m),   s_j = q . k_j,   c = scale * log2(e),
// one pass over the keys with a running reference m and sum.  A wave takes tiles of 32 keys, whose codes come through a ring in LDS (kv_tiles.h).  The
// keys, then the values, are the first operand of the two products, so that a lane has the scores of one query row, and the order of the keys
// and channels inside the products, which is free, is chosen so that the probabilities are the second product's second operand in the registers they are
// formed in.  A conversion of codes to bf16 is exact; it gives two channels of one key where the second product takes two keys of one channel: a
// byte permutation per two values.
//
// Few rows (Narrow, 16 or 32 at a time): the four waves of a work-group take every fourth tile of the same rows and meet in LDS at the end.  Bound by the cache's way from
// memory: 64 tokens over 500 - 8 192, 304 MB, 69 us, 4.4 TB/s, the way of the first tiles and the uneven ends included (64 channels, 152 MB: 43 us; 256, 304 MB: 71).
// More (Wide): each of four or eight waves has 32 rows of its own, the values are converted once for all of them.  Bound by the matrix cores and the vector
// instructions between them, and by the clock that the card keeps meanwhile.
// The work is dealt out by kv_deal.h: a work-group takes a run of tiles that may begin and end inside a block of rows; what it has of such a
// block goes to the workspace, and merge_kernel joins the pieces.
#pragma once

#include <type_traits>

#include "kv_deal.h"
#include "kv_format.h"
#include "kv_rows.h"
#include "kv_tiles.h"

namespace mars {
namespace kv {

constexpr float kFloor = -3.402823466e38f;  // the reference before the first key that counts: the least number, so that all scores pass it
constexpr float kSlack = 8.0f;              // how far (in powers of two) scores may pass the reference before it is moved up
// exp2(c s - m) is formed without rounding c s, so that the key that m is of gives 2 to what m was rounded by.  Beyond this (2^24) that is half a power of two and
// more, at 2^31 all of the exponent's range: there c s is rounded first, as m was, and the largest scores are the reference exactly.
constexpr float kLarge = 16777216.0f;
__device__ __forceinline__ bool any_large(float m) { return __any(__builtin_fabsf(m) > kLarge && m != kFloor); }
enum { KEYS = 0, ROWS = 1 };          // what the waves of a work-group divide between them

// (Written out: fmaxf would first quiet each operand.  The compiler does not wait for a matrix instruction's results in front of it: `a` comes from an
// operation of its own on the same results.)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
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

// Two keys' values of the same channel beside each other: the low halves of two conversions, or the high ones.
__device__ __forceinline__ u32 low_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ u32 high_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// The queries, as the first product's second operand, are bf16 rows as they are; fp32 rows are three bf16 terms, as the probabilities then are.  The
// probabilities of bf16 rows are one term, which is a choice: results are 0.0023 from 64 bits, of which their own rounding is 0.0017.  A second term would
// leave that alone, and cost 4 % with 64 tokens, 7 % with one, 15 % with 28 rows and 29 - 37 % where a wave has 32.  The sum l is that of the unrounded
// ones, since lse is its logarithm; where all probabilities of a row are equal they are rounded the same way, and the row is off by up to that one rounding.
// (Another sum, of the rounded ones, to divide by: 7 - 10 % with 32 rows per wave.)  The matrix cores also take codes and scales as they are, by queries of 8 bits: two
// such terms hold a bf16 number, and the conversion of the keys falls away (a tenth of the time with long caches, nothing with few rows).  But
// products of one instruction 2^16 below the largest are dropped there, and scores of 100 came out 1e-3 off; so it is not used.
typedef float f32x16 __attribute__((ext_vector_type(16)));

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

// log of the sum of exponentials that l counts against the reference m.
__device__ __forceinline__ float log_sum(float m, float l) { return l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f; }

// A row of the block of nodes from node0 on: the `row`-th of `rows`, node by node, a cache head's query heads beside each other.
template <typename T> struct RowOf {
  int node, head;            // node < 0: there is no such row
  unsigned long long word;   // its mask, where that is one word
  const T* q;                // (where there is no row: the block's first)
  __device__ __forceinline__ RowOf(const AttnArgs& a, int b, int cache_head, int node0, int row, int rows) {
    const bool live = row < rows;
    const int in = live ? row / a.group : 0;
    node = node0 + in;
    head = cache_head * a.group + (live ? row - in * a.group : 0);
    word = a.mask && a.words == 1 ? a.mask[static_cast<size_t>(b) * a.N + node] : 0;
    q = static_cast<const T*>(a.q) + b * a.q_request + static_cast<long>(node) * a.q_node + static_cast<long>(head) * a.q_head;
    if (!live) node = -1;
  }
};
// Where the results of a lane go: element [f][i] of its row among the 16 from `row0` on is channel (4g + i) * D/16 + f0 + f.
template <int D, int F, typename T>
__device__ __forceinline__ void write_narrow(const AttnArgs& a, int b, int head, int node0, int row0, int rows, int f0, const f32x4 (&o)[F], float m, float l) {
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
    a.lse[(static_cast<size_t>(b) * a.N + node) * a.q_heads + h] = log_sum(m, l);
}

// ---------------------------------------------------------------- 16 rows per lane column
// Both products on v_mfma_f32_16x16x32_bf16.  Lane (r = l % 16, g = l / 16):
//   scores    first operand: row r of a block of 16 keys, a quarter of its channels.  Row 4g + i of block b is the tile's key 8g + 4b + i, so that the lane
//             ends up with the scores of the eight keys 8g .. 8g + 7 for its query, in order --
//   values    -- which is what the second product's second operand holds.  Its first one: eight keys 8g .. 8g + 7 of D/16 channels of its own.
// What a lane has of a tile, in registers: sixteen keys' quarter twice, and eight keys' values.
template <int D> struct Keys16 {
  u32 k[2][D / 32], ks[2];
  __device__ __forceinline__ explicit Keys16(const uint8_t* tile) {
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
template <int D> struct Values16 {
  u32 v[Tile<D>::VW];
  u32x2 vs;
  __device__ __forceinline__ explicit Values16(const uint8_t* tile) {
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

template <int D, int RB, typename T> struct Queries16 {
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
  __device__ __forceinline__ void scores(const Keys16<D>& x, f32x4 (&sc)[2][RB]) const {
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
template <int D_, int RB, typename T_> struct Narrow {
  using T = T_;
  using Keys = Keys16<D_>;
  static constexpr int D = D_, MODE = KEYS, kRows = 16 * RB, kGroupWaves = kWaves;
  static constexpr int NF = D / 16;             // blocks of 16 channels of the result
  static constexpr int kParts = RB * NF;        // of a wave's result, four numbers of a lane each
  static constexpr int TERMS = std::is_same<T, float>::value ? 3 : 1;
  Queries16<D, RB, T> q;
  f32x4 o[RB][NF];                              // [f][i]: channel (4g + i) D/16 + f
  float m[RB], l[RB];
  bool large;                                   // (the same for the wave) a reference beyond kLarge
  int node[RB];                                 // of this lane's rows; < 0: no row
  unsigned long long word[RB];                  // the row's mask, where it is one word

  // Rows row0 .. of the block of nodes from node0 on, which has `rows`.
  __device__ __forceinline__ void start(const AttnArgs& a, int b, int head, int node0, int row0, int rows) {
    const int r = threadIdx.x % 16;
    large = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const RowOf<T> row(a, b, head, node0, row0 + rb * 16 + r, rows);
      node[rb] = row.node;
      word[rb] = row.word;
      q.load(rb, row.q, row.node >= 0);
      m[rb] = kFloor;
      l[rb] = 0.0f;
#pragma unroll
      for (int f = 0; f < NF; ++f) o[rb][f] = f32x4{0, 0, 0, 0};
    }
  }
  // One tile.  `plain` (the same for the wave): every row sees all of it, and all of it is there.  Otherwise: request b has n nodes behind
  // `len` tokens, the tile begins at t0; `bad`: which of its octets have no page.
  __device__ __forceinline__ void tile(const AttnArgs& a, const uint8_t* at, bool plain, int b, int len, int n, int t0, u32 bad) {
    const float c = a.scale_log2;
    const int g = threadIdx.x % kWave / 16;
    Values16<D> values(at);
    f32x4 sc[2][RB];
    q.scores(Keys16<D>(at), sc);
    __builtin_amdgcn_sched_barrier(0);  // (the values' conversions would be brought up to here, and their results kept)
    if (!plain) {
      const int first = t0 + g * 8 - len;
      const bool poison = bad >> g & 1;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const u32 sees = node[rb] < 0 ? 0u : seen(a, word[rb], b, node[rb], n, first);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float s = poison ? __builtin_nanf("") : sc[k][rb][i];
            sc[k][rb][i] = sees >> (4 * k + i) & 1 ? s : -__builtin_inff();
          }
      }
      values.cut(poison ? 0 : n - first);
    }
    float top[RB];
    bool up = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float t = fmaxf(sc[0][rb][0], sc[1][rb][0]);
      t = max3(t, sc[0][rb][1], sc[0][rb][2]);
      t = max3(t, sc[0][rb][3], sc[1][rb][1]);
      t = max3(t, sc[1][rb][2], sc[1][rb][3]);
      top[rb] = t * c;
      up |= top[rb] > m[rb] + kSlack;
    }
    if (__any(up)) {  // seldom after the first tiles
      large = false;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        float t = fmaxf(top[rb], __shfl_xor(top[rb], 16));
        t = fmaxf(m[rb], fmaxf(t, __shfl_xor(t, 32)));
        const float shrink = __builtin_amdgcn_exp2f(m[rb] - t);
        m[rb] = t;
        large |= any_large(t);
        l[rb] *= shrink;
#pragma unroll
        for (int f = 0; f < NF; ++f) o[rb][f] *= shrink;
      }
    }
    const float before = large ? c : 1.0f, factor = large ? 1.0f : c;  // (a branch instead would cost registers that four waves per SIMD do not have)
    u32 p[TERMS][RB][4];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(sc[h / 2][rb][h % 2 * 2] * before, factor, -m[rb]));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(sc[h / 2][rb][h % 2 * 2 + 1] * before, factor, -m[rb]));
        l[rb] += e0 + e1;
        u32 t[TERMS];
        split_pair<TERMS>(e0, e1, t);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) p[k][rb][h] = t[k];
      }
    __builtin_amdgcn_sched_barrier(0);
    values.each([&](int f, bf16x8 v) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t)
          o[rb][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, as_bf16x8(p[t][rb][0], p[t][rb][1], p[t][rb][2], p[t][rb][3]), o[rb][f], 0, 0, 0);
    });
  }
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      l[rb] += __shfl_xor(l[rb], 16);
      l[rb] += __shfl_xor(l[rb], 32);
    }
  }
  // The four waves' results for the same rows to wave 0.  sh: room for two waves' results; sh_m, sh_l: [4][kRows].
  __device__ __forceinline__ void join(f32x4* sh_o, float* sh_m, float* sh_l) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane % 16;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
      if (lane < 16) {
        sh_m[wave * kRows + rb * 16 + r] = m[rb];
        sh_l[wave * kRows + rb * 16 + r] = l[rb];
      }
    __syncthreads();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float all = kFloor, sum = 0.0f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) all = fmaxf(all, sh_m[v * kRows + rb * 16 + r]);
#pragma unroll
      for (int v = 0; v < kWaves; ++v) sum += sh_l[v * kRows + rb * 16 + r] * __builtin_amdgcn_exp2f(sh_m[v * kRows + rb * 16 + r] - all);
      const float shrink = __builtin_amdgcn_exp2f(m[rb] - all);
#pragma unroll
      for (int f = 0; f < NF; ++f) o[rb][f] *= shrink;
      m[rb] = all;
      l[rb] = sum;
    }
    // waves 2 and 3 to 0 and 1, then 1 to 0
#pragma unroll
    for (int half = 2; half >= 1; half >>= 1) {
      f32x4* const sh = sh_o + (wave & (half - 1)) * (kParts * kWave) + lane;
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) sh[i * kWave] = o[i / NF][i % NF];
      }
      __syncthreads();
      if (wave < half) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) o[i / NF][i % NF] += sh[i * kWave];
      }
      __syncthreads();
    }
  }
  __device__ __forceinline__ void write(const AttnArgs& a, int b, int head, int node0, int row0, int rows) const {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) write_narrow<D, NF, T>(a, b, head, node0, row0 + rb * 16, rows, 0, o[rb], m[rb], l[rb]);
  }
  template <typename P> __device__ __forceinline__ void save(const P& piece) const {
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
      if (lane < 16) {
        piece.reference(rb * 16 + lane) = m[rb];
        piece.sum(rb * 16 + lane) = l[rb];
      }
#pragma unroll
    for (int i = 0; i < kParts; ++i) piece.part(i, lane) = o[i / NF][i % NF];
  }
  // Joining pieces: kStrips times a wave takes a quarter of the parts of kStripRows rows.
  static constexpr int kStrips = RB, kStripRows = 16, kQuarter = NF / 4;
  __device__ static __forceinline__ int strip_row(int strip) { return strip * 16 + threadIdx.x % 16; }  // of the lane, in the wave's rows
  __device__ static __forceinline__ int strip_wave(int) { return 0; }                                    // whose piece
  __device__ static __forceinline__ int strip_part(int strip, int quarter, int i) { return strip * NF + quarter * kQuarter + i; }
  __device__ static __forceinline__ void write_quarter(const AttnArgs& a, int b, int head, int node0, int strip, int rows, int quarter, const f32x4 (&x)[kQuarter],
                                                       float m, float l) {
    write_narrow<D, kQuarter, T>(a, b, head, node0, strip * 16, rows, quarter * kQuarter, x, m, l);
  }
};

// ---------------------------------------------------------------- 32 rows per wave
// Both products on v_mfma_f32_32x32x16_bf16, which holds the vector port for 12 of its 32 clocks, that of 16 rows for 10 of 16.  Lane (r = l % 32, h = l / 32):
//   scores    first operand: key r of the tile, half of its channels.  The lane ends up with the scores of keys 8a + 4h + i, i < 4, for its query --
//   values    -- which are eight keys each of the second product's two steps: keys 16t + 4h .. + 3 and 8 more on.  Its first operand: the same keys of D/32 channels.
// The waves of a work-group go through the tiles together, each converts the values of 16 keys of the next step for all of them, and waits for the others once per
// step (64 keys for four waves, 128 for eight, of which one work-group fills a compute unit; two of four end 20% apart, as one is served first throughout).
// 4 trees of 208 rows over 60 000 - 131 000 tokens: 410 us (0.83 PFLOP/s, 0.9 with the rows that fill up the last wave's 32; a large library product reaches
// 1.2), by work-groups of four waves 480, by waves of 64 rows, one per SIMD, 580.  16 trees of 240 rows over 1 024 - 8 191: 107 us, by four 118.  The matrix
// cores are busy for 30 to 40 % of the clocks, of which there are 2.0 to 2.2 GHz under this load.  fp32 rows (four waves) take three times the products, and their terms of the
// queries, 96 registers with 128 channels and 192 with 256, leave too few: 32 - 96 and 252 - 312 bytes of a lane are spilled.  16 trees of 240 rows over 1 024 - 8 191: 223 us
// (bf16 111); four heads of 256 channels 445 (bf16 151).  Scores a tile ahead, the exponentials laid between the matrix instructions,
// priorities and a deeper ring changed nothing or cost a little.
template <int D> struct Keys32 {
  u32 k[D / 64][4], ks[D / 64];  // 32 channels each, 64 s + 32 h
  Keys32() = default;
  __device__ __forceinline__ explicit Keys32(const uint8_t* tile) {
    using X = Tile<D>;
    const u32 lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
#pragma unroll
    for (int s = 0; s < D / 64; ++s) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(tile + X::key_slot(r, 2 * s + h) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) k[s][j] = w[j];
      ks[s] = tile[2 * X::kCodes + r * (D / 32) + 2 * s + h];
    }
  }
};
template <int D> struct Values32 {
  static constexpr int C = D / 32;  // channels of a lane: C r ..
  u32 v[2][4], vs[2];               // of octet 2t + o: tokens 4h .. 4h + 3, a dword column's codes, their scales
  __device__ __forceinline__ Values32(const uint8_t* tile, u32 t) {
    using X = Tile<D>;
    const u32 lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
#pragma unroll
    for (u32 o = 0; o < 2; ++o) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(tile + X::kCodes + X::value_slot(2 * t + o, r * C / 8, h) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[o][j] = w[j];
      vs[o] = *reinterpret_cast<const u32*>(tile + 2 * X::kCodes + (D <= 128 ? 128 : 256) + (2 * t + o) * (D / 4) + r * C / 32 * 8 + 4 * h);
    }
  }
  // Only the first `there` of the step's 16 tokens count, and none of its octets in `bad`: elsewhere memory holds anything, and 0 times that has to be 0.
  __device__ __forceinline__ void cut(int there, u32 bad) {
    const int h = threadIdx.x % kWave / 32;
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      const int n = bad >> o & 1 ? 0 : there - 8 * o - 4 * h;
      vs[o] = n >= 4 ? vs[o] : n <= 0 ? 0 : vs[o] & ((1u << (8 * n)) - 1);
    }
  }
  // f(block, fragment) for the C blocks: channel C r + block.
  template <typename F> __device__ __forceinline__ void each(F f) const {
    const u32 shift = D == 64 ? (threadIdx.x & 3) * 8 : D == 128 ? (threadIdx.x & 1) * 16 : 0;
    u32 w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = v[j / 4][j % 4] >> shift;
    const u32 s[8] = {scale_at<0>(vs[0]), scale_at<1>(vs[0]), scale_at<2>(vs[0]), scale_at<3>(vs[0]),
                      scale_at<0>(vs[1]), scale_at<1>(vs[1]), scale_at<2>(vs[1]), scale_at<3>(vs[1])};
    auto pair = [&](auto byte) {
      constexpr int BYTE = decltype(byte)::value;
      u32 y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = decode<BYTE>(w[j], s[j]);
      f(2 * BYTE, as_bf16x8(low_halves(y[0], y[1]), low_halves(y[2], y[3]), low_halves(y[4], y[5]), low_halves(y[6], y[7])));
      f(2 * BYTE + 1, as_bf16x8(high_halves(y[0], y[1]), high_halves(y[2], y[3]), high_halves(y[4], y[5]), high_halves(y[6], y[7])));
    };
    pair(std::integral_constant<int, 0>{});
    if constexpr (C > 2) pair(std::integral_constant<int, 1>{});
    if constexpr (C > 4) {
      pair(std::integral_constant<int, 2>{});
      pair(std::integral_constant<int, 3>{});
    }
  }
};

template <int D, typename T> struct Queries32 {
  static constexpr int S = D / 16, TERMS = std::is_same<T, float>::value ? 3 : 1;  // steps of 16 channels
  bf16x8 q[TERMS][S];
  __device__ __forceinline__ void load(const T* row, bool live) {
    const int h = threadIdx.x % kWave / 32;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      u32 t[4][TERMS];
      const Eight e = load_eight(row + s / 4 * 64 + h * 32 + s % 4 * 8);
#pragma unroll
      for (int p = 0; p < 4; ++p) split_pair<TERMS>(live ? e.x[2 * p] : 0.0f, live ? e.x[2 * p + 1] : 0.0f, t[p]);
#pragma unroll
      for (int k = 0; k < TERMS; ++k) q[k][s] = as_bf16x8(t[0][k], t[1][k], t[2][k], t[3][k]);
    }
  }
  __device__ __forceinline__ f32x16 scores(const Keys32<D>& x) const {
    f32x16 sc = {};
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const u32 scale = scale_at<0>(x.ks[s / 4]), w = x.k[s / 4][s % 4];
      const bf16x8 k = as_bf16x8(decode<0>(w, scale), decode<1>(w, scale), decode<2>(w, scale), decode<3>(w, scale));
#pragma unroll
      for (int t = TERMS - 1; t >= 0; --t) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[t][s], sc, 0, 0, 0);
    }
    return sc;
  }
};

// Where a quarter of a lane's results goes: [block][i] is channel C (8 quarter + 4 h + i) + block of its row.
template <int D, typename T>
__device__ __forceinline__ void write_wide(const AttnArgs& a, int b, int head, int node0, int row0, int rows, int quarter, const f32x4 (&o)[D / 32], float m, float l) {
  constexpr int C = D / 32;
  const int lane = threadIdx.x % kWave, h = lane / 32, row = row0 + lane % 32;
  if (row >= rows) return;
  const int in = row / a.group, node = node0 + in, q_head = head * a.group + row - in * a.group;
  const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
  T* at = static_cast<T*>(a.out) + b * a.out_request + node * a.out_node + q_head * a.out_head + C * (8 * quarter + 4 * h);
  float x[4 * C];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int k = 0; k < C; ++k) x[i * C + k] = o[k][i] * inverse;
#pragma unroll
  for (int i = 0; i < 4 * C; i += 8) {
    if constexpr (std::is_same<T, float>::value) {
      *reinterpret_cast<f32x4*>(at + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
      *reinterpret_cast<f32x4*>(at + i + 4) = f32x4{x[i + 4], x[i + 5], x[i + 6], x[i + 7]};
    } else {
      *reinterpret_cast<u32x4*>(at + i) = u32x4{round_pair(x[i], x[i + 1]), round_pair(x[i + 2], x[i + 3]), round_pair(x[i + 4], x[i + 5]), round_pair(x[i + 6], x[i + 7])};
    }
  }
  if (a.lse && h == 0 && quarter == 0) a.lse[(static_cast<size_t>(b) * a.N + node) * a.q_heads + q_head] = log_sum(m, l);
}

template <int D_, typename T_, int WAVES> struct Wide {
  using T = T_;
  static constexpr int D = D_, MODE = ROWS, kRows = 32, kGroupWaves = WAVES;
  static constexpr int C = D / 32;              // blocks of 32 channels of the result
  static constexpr int kParts = 4 * C;          // four numbers of a lane each
  static constexpr int TERMS = std::is_same<T, float>::value ? 3 : 1;
  Queries32<D, T> q;
  Keys32<D> next;                               // of the next tile
  f32x16 o[C];                                  // [block][i]: channel C (8 (i/4) + 4h + i%4) + block
  float m, l;
  bool large;                                   // (the same for the wave) a reference beyond kLarge
  int node;                                     // of this lane's row; < 0: no row
  unsigned long long word;

  __device__ __forceinline__ void start(const AttnArgs& a, int b, int head, int node0, int row0, int rows) {
    const RowOf<T> row(a, b, head, node0, row0 + threadIdx.x % 32, rows);
    node = row.node;
    word = row.word;
    q.load(row.q, node >= 0);
    m = kFloor;
    l = 0.0f;
    large = false;
#pragma unroll
    for (int k = 0; k < C; ++k) o[k] = f32x16{};
  }
  // A step's values as operands, to `values` [tile][2 C][64]: 16 keys' by each wave.  `tiles`: the step's, keys t0 ..
  __device__ __forceinline__ static void convert(const uint8_t* tiles, u32x4* values, const u32* sh_bad, int t0, int end) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const u32 bad = __builtin_amdgcn_readfirstlane(sh_bad[wave / 2]) >> (wave % 2 * 2);
    t0 += wave * 16;
    Values32<D> x(tiles + wave / 2 * Tile<D>::kBytes, wave % 2);
    if (t0 + 16 > end || (bad & 3)) x.cut(end - t0, bad);
    u32x4* const at = values + wave * C * kWave + threadIdx.x % kWave;
    x.each([&](int k, bf16x8 v) { at[k * kWave] = __builtin_bit_cast(u32x4, v); });
  }
  __device__ __forceinline__ void begin(const uint8_t* tile) { next = Keys32<D>(tile); }
  // A tile (as Narrow::tile says), its values as operands at `values`; the next one is at `after`.
  __device__ __forceinline__ void tile(const AttnArgs& a, const uint8_t* after, const u32x4* values, u32 bad, int b, int len, int n, int t0) {
    const float c = a.scale_log2;
    f32x16 s = q.scores(next);
    if (t0 + kTile > len || bad) {
      const int h = threadIdx.x % kWave / 32;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const u32 sees = node < 0 ? 0u : seen(a, word, b, node, n, t0 + 8 * k - len) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = bad >> k & 1 ? __builtin_nanf("") : s[4 * k + i];
          s[4 * k + i] = sees >> i & 1 ? x : -__builtin_inff();
        }
      }
    }
    float top = fmaxf(s[0], s[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) top = max3(top, s[i], s[i + 1]);
    top *= c;
    if (__any(top > m + kSlack)) {  // seldom after the first tiles
      top = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)));
      const float shrink = __builtin_amdgcn_exp2f(m - top);
      m = top;
      large = any_large(m);
      l *= shrink;
#pragma unroll
      for (int k = 0; k < C; ++k) o[k] *= shrink;
    }
    float factor = c;
    if (large) {
      s *= c;
      factor = 1.0f;
    }
    next = Keys32<D>(after);  // (5% faster here than in front of the branches)
    u32 p[TERMS][2][4];  // probabilities, in terms, of the two steps of the product with the values
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float e0 = __builtin_amdgcn_exp2f(fmaf(s[2 * i], factor, -m)), e1 = __builtin_amdgcn_exp2f(fmaf(s[2 * i + 1], factor, -m));
      l += e0 + e1;
      u32 x[TERMS];
      split_pair<TERMS>(e0, e1, x);
#pragma unroll
      for (int k = 0; k < TERMS; ++k) p[k][i / 4][i % 4] = x[k];
    }
    u32x4 v[2 * C];
    auto load = [&](int k) { v[k] = values[k * kWave + threadIdx.x % kWave]; };
    load(0);
    load(1);
#pragma unroll
    for (int i = 0; i < 2 * C; ++i) {
      const int t = i / C, k = i % C;
      if (i + 2 < 2 * C) load(i + 2);
#pragma unroll
      for (int x = TERMS - 1; x >= 0; --x)
        o[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[i]), as_bf16x8(p[x][t][0], p[x][t][1], p[x][t][2], p[x][t][3]), o[k], 0, 0, 0);
    }
  }
  __device__ __forceinline__ void finish() { l += __shfl_xor(l, 32); }
  __device__ __forceinline__ f32x4 part(int i) const { return f32x4{o[i / 4][i % 4 * 4], o[i / 4][i % 4 * 4 + 1], o[i / 4][i % 4 * 4 + 2], o[i / 4][i % 4 * 4 + 3]}; }
  __device__ __forceinline__ void write(const AttnArgs& a, int b, int head, int node0, int row0, int rows) const {
#pragma unroll
    for (int quarter = 0; quarter < 4; ++quarter) {
      f32x4 x[C];
#pragma unroll
      for (int k = 0; k < C; ++k) x[k] = part(4 * k + quarter);
      write_wide<D, T>(a, b, head, node0, row0, rows, quarter, x, m, l);
    }
  }
  template <typename P> __device__ __forceinline__ void save(const P& piece) const {
    const int lane = threadIdx.x % kWave;
    if (lane < 32) {
      piece.reference(lane) = m;
      piece.sum(lane) = l;
    }
#pragma unroll
    for (int i = 0; i < kParts; ++i) piece.part(i, lane) = part(i);
  }
  static constexpr int kStrips = WAVES, kStripRows = 32, kQuarter = C;
  __device__ static __forceinline__ int strip_row(int) { return threadIdx.x % 32; }
  __device__ static __forceinline__ int strip_wave(int strip) { return strip; }
  __device__ static __forceinline__ int strip_part(int, int quarter, int i) { return 4 * i + quarter; }
  __device__ static __forceinline__ void write_quarter(const AttnArgs& a, int b, int head, int node0, int strip, int rows, int quarter, const f32x4 (&x)[C], float m,
                                                       float l) {
    write_wide<D, T>(a, b, head, node0, strip * 32, rows, quarter, x, m, l);
  }
};

// ---------------------------------------------------------------- kernels
// A wave's piece in the workspace: its rows' references, their sums, then the results lane by lane.
template <typename W> struct Piece {
  static constexpr int kFloats = 2 * W::kRows + W::kParts * 256;
  float* at;
  __device__ __forceinline__ Piece(float* partial, long slot) : at(partial + slot * kFloats) {}
  __device__ __forceinline__ float& reference(int row) const { return at[row]; }
  __device__ __forceinline__ float& sum(int row) const { return at[W::kRows + row]; }
  __device__ __forceinline__ f32x4& part(int i, int lane) const { return reinterpret_cast<f32x4*>(at + 2 * W::kRows)[i * kWave + lane]; }
};

// Rows that see nothing because their request has fewer nodes (or no sequence): zeros, by one work-group per request in front of its share of the attention.  That is
// what ragged prompts are bound by: 8 with 100 to 2 048 of N = 2 048 nodes behind up to 100 tokens 640 us, with 100 each 510, with all of them 450.
template <typename T, int D> __device__ __forceinline__ void clear_rows(const AttnArgs& a, int b, int n) {
  const long items = static_cast<long>(a.N - n) * a.q_heads * (D / 8);
  for (long i = threadIdx.x; i < items; i += blockDim.x) {
    const int c = static_cast<int>(i % (D / 8)), h = static_cast<int>(i / (D / 8) % a.q_heads), node = n + static_cast<int>(i / (D / 8) / a.q_heads);
    T* at = static_cast<T*>(a.out) + b * a.out_request + node * a.out_node + h * a.out_head + c * 8;
    const u32 none[4] = {0, 0, 0, 0};
    store_eight(at, none);
    if (c == 0 && a.lse) a.lse[(static_cast<size_t>(b) * a.N + node) * a.q_heads + h] = -__builtin_inff();
  }
}

// Work-groups that have to fit a compute unit beside each other: what the compiler may give a wave of registers, and the ring of LDS.
// 16 rows of bf16 fit the 128 registers of four waves per SIMD where a tile lies in one page (uniform): 64 tokens over 500 - 8 192 67 us, three 72; where it does not,
// pages of 16 tokens 99 and 73.
constexpr int per_unit(int D, int mode, int waves, int rows, bool f32, bool uniform) {
  if (mode == KEYS) return (D == 256 ? 1 : 2) + (rows == 16 && !f32 ? (D <= 128 && uniform ? 2 : 1) : 0);
  return D == 256 || waves > kWaves ? 1 : 2;
}
template <typename W, bool UNIFORM>
constexpr int kPerUnit = per_unit(W::D, W::MODE, W::kGroupWaves, W::kRows, std::is_same<typename W::T, float>::value, UNIFORM);
template <typename W> constexpr int kValuesBytes = W::MODE == ROWS ? W::kGroupWaves * W::D * 64 : 16;  // of two steps' values as operands
template <typename W, bool UNIFORM> constexpr int stages_of() {  // units in the ring, those that are worked on among them
  constexpr int n = (160 * 1024 / kPerUnit<W, UNIFORM> - 1024 - kValuesBytes<W>) / (kWaves * Tile<W::D>::kBytes);
  return n > 4 ? 4 : n;
}

template <typename W, bool UNIFORM>
__global__ void __launch_bounds__(W::kGroupWaves * kWave, (kPerUnit<W, UNIFORM> * W::kGroupWaves / kWaves)) attention_kernel(AttnArgs a) {
  constexpr int D = W::D, MODE = W::MODE, GROUP = W::kGroupWaves, STAGES = stages_of<W, UNIFORM>();
  // Units in flight behind the one that is waited for (in mode ROWS a step is half a unit, or a whole one by eight waves):
  constexpr int AHEAD = GROUP > kWaves ? STAGES - 3 : STAGES - 2;
  using X = Tile<D>;
  static_assert(AHEAD >= 0, "a unit in flight while another is worked on");
  constexpr int kJoin = MODE == KEYS ? 2 * W::kParts * 1024 : 0;  // bytes for two waves' results
  constexpr int kRing = STAGES * kWaves * X::kBytes;
  __shared__ __attribute__((aligned(1024))) uint8_t sh_ring[kRing > kJoin ? kRing : kJoin];
  __shared__ __attribute__((aligned(16))) u32x4 sh_values[kValuesBytes<W> / 16];
  __shared__ u32 sh_bad[STAGES][kWaves];
  __shared__ float sh_m[MODE == KEYS ? kWaves * W::kRows : 1], sh_l[MODE == KEYS ? kWaves * W::kRows : 1];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;

  if (a.n_new || a.seqs || a.B > a.c.sequences)  // (otherwise every request has N nodes)
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
      const int n = Request(a, b).n;
      if (n < a.N) clear_rows<typename W::T, D>(a, b, n);
    }
  Deal deal(a, gridDim.x);
  if (deal.total == 0) return;
  const u32 share = deal.share;
  // neighbours in the deal on the same die (block index mod 8), all dies alike
  const u32 per_die = ((deal.total + share - 1) / share + 7) >> 3;
  if (blockIdx.x >> 3 >= per_die) return;
  const u32 group = (blockIdx.x & 7) * per_die + (blockIdx.x >> 3);
  const unsigned long long my_begin = static_cast<unsigned long long>(group) * share;
  if (my_begin >= deal.total) return;
  const u32 unit0 = static_cast<u32>(my_begin), unit1 = static_cast<u32>(min(my_begin + share, static_cast<unsigned long long>(deal.total)));
  const u32 ring = lds_address(sh_ring);

  W w;
  for (u32 u = unit0; u < unit1;) {
    const auto p = deal.find(u);
    if (p.count == 0) {
      u += p.offset;
      continue;
    }
    const u32 taken = min(p.count - p.offset, unit1 - u);
    const bool whole = taken == p.count;
    const int units = static_cast<int>(deal.whole ? p.r.block_units(a, p.block) : taken);
    const int node0 = p.block * a.nodes, rows = min(a.nodes, p.r.n - node0) * a.group, row0 = MODE == ROWS ? wave * W::kRows : 0;
    const int len = p.r.len, n = p.r.n, end = len + n;
    // no row of this wave sees keys from here on (0: it has no rows)
    const int limit = row0 >= rows ? 0 : a.mask ? end : len + 1 + node0 + (min(rows, row0 + W::kRows) - 1) / a.group;
    const int from = static_cast<int>(p.offset) * kUnit;
    // (in front of the queries' loads; LDS is free: the piece before ended with a barrier)
    Fetch<D, UNIFORM> fetch(a, sequence_of(a.c, a.seqs, p.b), p.head, end, from + wave % kWaves * kTile);
    u32 stage = 0;
    auto issue = [&](u32 to) {
      const u32 bad = fetch.next(ring + (to * kWaves + wave) * X::kBytes);
      if (lane == 0) sh_bad[to][wave] = bad;
    };
#pragma unroll
    for (int i = 0; i <= AHEAD; ++i)
      if (i < units && wave < kWaves) issue(i);
    w.start(a, p.b, p.head, node0, row0, rows);

    // This wave's tile of a unit, in place `at` of the ring, is there; with a barrier (which leaves alone what is in flight from memory) those of others, and everybody
    // is done with the step before.
    auto wait_for = [&](int unit) {
      if (unit + AHEAD < units) arrived<AHEAD * X::kLoads>();
      else arrived<0>();
    };
    auto issue_behind = [&](int unit, u32 at) {
      if (unit + AHEAD + 1 < units) issue(at + AHEAD + 1 >= STAGES ? at + AHEAD + 1 - STAGES : at + AHEAD + 1);
    };
    if constexpr (MODE == KEYS) {
      for (int unit = 0; unit < units; ++unit) {
        wait_for(unit);
        issue_behind(unit, stage);
        const int t0 = from + unit * kUnit + wave * kTile;
        if (t0 < limit) {
          const u32 bad = __builtin_amdgcn_readfirstlane(sh_bad[stage][wave]);
          w.tile(a, sh_ring + (stage * kWaves + wave) * X::kBytes, t0 + kTile <= len && bad == 0, p.b, len, n, t0, bad);
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
      }
    } else {
      // While a step is worked on, the values of the next one are converted.  Its tiles are those that two of four waves have fetched, or four of eight; the
      // places of the step before are the same waves', to be filled again.
      constexpr int TILES = GROUP / 2;
      u32x4 *here = sh_values, *there = sh_values + kValuesBytes<W> / 32;
      int t0 = from;
      auto next_step = [&](int unit, u32 at, int first) {
        const bool mine = wave >= first && wave < first + TILES;
        if (mine) wait_for(unit);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (mine) issue_behind(unit, at);
      };
      auto step = [&](const uint8_t* now, const u32* bad, const uint8_t* then, const u32* bad_then) {
        W::convert(then, there, bad_then, t0 + TILES * kTile, end);
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          if (t0 < limit)
            w.tile(a, i + 1 < TILES ? now + (i + 1) * X::kBytes : then, here + i * (D / 16) * kWave, __builtin_amdgcn_readfirstlane(bad[i]), p.b, len, n, t0);
          t0 += kTile;
        }
        u32x4* const done = here;
        here = there;
        there = done;
      };
      next_step(0, 0, 0);
      W::convert(sh_ring, here, sh_bad[0], t0, end);
      w.begin(sh_ring);
      for (int unit = 0; unit < units; ++unit) {
        const uint8_t* const now = sh_ring + stage * kWaves * X::kBytes;
        const u32* const bad = sh_bad[stage];
        const u32 following = stage + 1 == STAGES ? 0 : stage + 1;
        const uint8_t* const then = sh_ring + following * kWaves * X::kBytes;
        if constexpr (GROUP > kWaves) {
          next_step(unit + 1, following, 0);
          step(now, bad, then, sh_bad[following]);
        } else {
          next_step(unit, stage, 2);
          step(now, bad, now + 2 * X::kBytes, bad + 2);
          next_step(unit + 1, following, 0);
          step(now + 2 * X::kBytes, bad + 2, then, sh_bad[following]);
        }
        stage = following;
      }
    }
    w.finish();
    __syncthreads();  // the ring is free
    if constexpr (MODE == KEYS) w.join(reinterpret_cast<f32x4*>(sh_ring), sh_m, sh_l);
    if (MODE == ROWS || wave == 0) {
      if (whole) w.write(a, p.b, p.head, node0, row0, rows);
      else  // the first piece of the group's run, or its last one
        w.save(Piece<W>(a.partial, (static_cast<long>(group) * 2 + (u == unit0 ? 0 : 1)) * (MODE == ROWS ? GROUP : 1) + (MODE == ROWS ? wave : 0)));
    }
    u += taken;
  }
}

// Joins the pieces of blocks that were dealt to several work-groups: one work-group for every place where the deal cuts one, of which the
// first of a block takes it; a wave per strip of rows and quarter of the result's channels, several pieces at a time under way (it is the latency of
// these loads that counts: a piece at a time took 8 us where this takes 4; 16 trees, 100 MB of pieces: 18 us).
template <typename W> __global__ void __launch_bounds__(kThreads) merge_kernel(AttnArgs a, u32 groups) {
  constexpr int F = W::kQuarter, AT_ONCE = F > 2 ? 4 : 8;
  Deal deal(a, groups);
  if (deal.whole || deal.total == 0) return;
  const u32 share = deal.share;
  const u32 cut = blockIdx.x + 1;
  const unsigned long long at = static_cast<unsigned long long>(cut) * share;
  if (at >= deal.total) return;
  const auto p = deal.find(static_cast<u32>(at));
  if (p.count == 0 || p.begin == at) return;          // cut between two blocks
  const u32 first = p.begin / share, last = (p.begin + p.count - 1) / share;
  if (cut != first + 1) return;                       // an earlier cut's
  const int node0 = p.block * a.nodes, rows = min(a.nodes, p.r.n - node0) * a.group;
  const int quarter = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  for (int strip = blockIdx.y; strip < W::kStrips && strip * W::kStripRows < rows; strip += gridDim.y) {
    const int row = W::strip_row(strip);
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
        const Piece<W> piece(a.partial, (static_cast<long>(x) * 2 + second) * (W::MODE == ROWS ? W::kGroupWaves : 1) + W::strip_wave(strip));
        pm[i] = piece.reference(row);
        pl[i] = piece.sum(row);
#pragma unroll
        for (int f = 0; f < F; ++f) po[i][f] = piece.part(W::strip_part(strip, quarter, f), lane);
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
    W::write_quarter(a, p.b, p.head, node0, strip, rows, quarter, o, m, l);
  }
}

}  // namespace kv
}  // namespace mars
