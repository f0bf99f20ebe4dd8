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
constexpr int kTile = 32;             // keys per wave and step
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

// The deal.  Request b has items[b] = heads x blocks of rows, each of tiles[b] units; units in front of it: begin.
template <int ROWS_PER_ITEM, int UNIT> struct Deal {
  int n, len, items, tiles;
  __device__ __forceinline__ Deal(const AttnArgs& a, int b) {
    const int s = sequence_of(a.c, a.seqs, b);
    n = a.n_new ? min(max(a.n_new[b], 0), a.N) : a.N;
    len = 0;
    if (s >= 0) len = min(max(a.c.lens[s], 0), a.c.width << a.c.log_page);
    else n = 0;
    const long rows = static_cast<long>(n) * a.group;
    items = a.c.heads * static_cast<int>((rows + ROWS_PER_ITEM - 1) / ROWS_PER_ITEM);
    tiles = (len + n + UNIT - 1) / UNIT;
  }
  __device__ __forceinline__ long units() const { return static_cast<long>(items) * tiles; }
};
// Units in front of every request, in LDS: sh[b], b <= B.  All threads of a work-group of kThreads.
template <typename D> __device__ __forceinline__ void deal_out(const AttnArgs& a, u32* sh) {
  __shared__ u32 sums[kThreads / kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  u32 front = 0;
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    const u32 v = b < a.B ? static_cast<u32>(D(a, b).units()) : 0;
    u32 x = v;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const u32 y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    if (lane == kWave - 1) sums[wave] = x;
    __syncthreads();
    u32 total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / kWave; ++w) {
      if (w < wave) x += sums[w];
      total += sums[w];
    }
    if (b < a.B) sh[b] = front + x - v;
    front += total;
    __syncthreads();
  }
  if (threadIdx.x == 0) sh[a.B] = front;
  __syncthreads();
}
// The request that unit u belongs to: the last b with sh[b] <= u (requests without units never are).
__device__ __forceinline__ int request_of(const u32* sh, int B, u32 u) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sh[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
__device__ __forceinline__ u32 share_of(u32 total, u32 groups, u32 least) { return max((total + groups - 1) / groups, least); }

// What a lane has of a tile, as it came from memory.
template <int D> struct Tile {
  static constexpr int S = D / 32, VW = D == 256 ? 16 : 8;
  u32 k[2][S], ks[2], v[VW];
  u32x2 vs;
};

// A wave's rows, their queries and what it has gathered for them.
template <int D, int RB, typename T> struct Wave {
  static constexpr int S = D / 32;              // steps of 32 channels
  static constexpr int NF = D / 16;             // blocks of 16 channels of the result
  static constexpr int TERMS = std::is_same<T, float>::value ? 3 : 1;
  bf16x8 q[TERMS][RB][S];
  f32x4 o[NF][RB];
  float m[RB], l[RB];
  int node[RB];                                 // of this lane's rows; < 0: no row

  __device__ __forceinline__ void start(const AttnArgs& a, int b, int head, int row0, int rows) {
    const int lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int row = row0 + rb * 16 + r;
      const bool live = row < rows;
      node[rb] = live ? row / a.group : -1;
      const T* at = static_cast<const T*>(a.q) + b * a.q_request + static_cast<long>(live ? node[rb] : 0) * a.q_node +
                    static_cast<long>(head * a.group + (live ? row - node[rb] * a.group : 0)) * a.q_head + g * (D / 4);
#pragma unroll
      for (int s = 0; s < S; ++s) {
        u32 t[4][TERMS];
        const Eight e = load_eight(at + s * 8);
#pragma unroll
        for (int p = 0; p < 4; ++p) split_pair<TERMS>(live ? e.x[2 * p] : 0.0f, live ? e.x[2 * p + 1] : 0.0f, t[p]);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) q[k][rb][s] = as_bf16x8(t[0][k], t[1][k], t[2][k], t[3][k]);
      }
      m[rb] = kFloor;
      l[rb] = 0.0f;
#pragma unroll
      for (int f = 0; f < NF; ++f) o[f][rb] = f32x4{0, 0, 0, 0};
    }
  }
};

// Where the lane finds its keys and values: requests' pages, one tile after the other.
template <int D> struct Reader {
  const AttnArgs& a;
  const int32_t* row;       // of the page table
  int head, end;            // keys there are
  __device__ __forceinline__ Reader(const AttnArgs& a_, int s, int head_, int end_)
      : a(a_), row(a_.c.page_table + static_cast<size_t>(s) * a_.c.width), head(head_), end(end_) {}
  // The page that holds position t (past the end: the last position); -1 past the table.
  __device__ __forceinline__ int page(int t) const {
    const int i = min(t, end - 1) >> a.c.log_page;
    return i < a.c.width ? row[i] : -1;
  }
  __device__ __forceinline__ void load(int t0, int kpage, int vpage, Tile<D>& x) const {
    const int lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
    const u32 in_page = (1u << a.c.log_page) - 1, last = static_cast<u32>(end - 1) & ~7u;
    const u32 kp = static_cast<u32>(kpage) < static_cast<u32>(a.c.pages) ? kpage : 0, vp = static_cast<u32>(vpage) < static_cast<u32>(a.c.pages) ? vpage : 0;
    const uint8_t* kb = head_of(a.c, a.layer_offset, kp, head);
    const u32 kt = (min(static_cast<u32>(t0) + (r >> 2) * 8, last) & in_page) + (r & 3);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint8_t* at = kb + Place<D>::key(kt + 4 * b) + g * (D / 8);
      if constexpr (D == 64) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(at);
        x.k[b][0] = w[0]; x.k[b][1] = w[1];
      } else {
#pragma unroll
        for (int i = 0; i < D / 128; ++i) {
          const u32x4 w = reinterpret_cast<const u32x4*>(at)[i];
#pragma unroll
          for (int j = 0; j < 4; ++j) x.k[b][4 * i + j] = w[j];
        }
      }
      const uint8_t* st = kb + Place<D>::key_scale(a.c.log_page, kt + 4 * b);
      if constexpr (D == 256) x.ks[b] = *reinterpret_cast<const uint16_t*>(st + 2 * g);
      else x.ks[b] = st[D == 64 ? g >> 1 : g];
    }
    const uint8_t* vb = head_of(a.c, a.layer_offset, vp, head);
    const u32 vt = min(static_cast<u32>(t0) + g * 8, last) & in_page;
    const u32 column = D == 64 ? r >> 1 : D == 128 ? r : 2 * r;
    const u32x4* at = reinterpret_cast<const u32x4*>(vb + Place<D>::value(a.c.log_page, vt) + column * 32);
#pragma unroll
    for (int i = 0; i < Tile<D>::VW / 4; ++i) {
      const u32x4 w = at[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) x.v[4 * i + j] = w[j];
    }
    x.vs = *reinterpret_cast<const u32x2*>(vb + Place<D>::value_scale(a.c.log_page, vt) + (r * (D / 16)) / 32 * 8);
  }
};

// Two keys' values of the same channel beside each other: the low halves of two conversions, or the high ones.
__device__ __forceinline__ u32 low_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ u32 high_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// `sees[rb]`: of keys 8g .. 8g + 7 of the tile, which the lane's row sees (bit by bit); only looked at where MASKED.
// `poison`: the lane's octet has no page.
template <int D, int RB, typename T, bool MASKED>
__device__ __forceinline__ void attend(Wave<D, RB, T>& w, const Tile<D>& x, float c, const u32 (&sees)[RB], int there, bool poison) {
  constexpr int S = D / 32, NF = D / 16, TERMS = Wave<D, RB, T>::TERMS;
  const int lane = threadIdx.x % kWave, r = lane % 16;
  f32x4 sc[2][RB];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) sc[b][rb] = f32x4{0, 0, 0, 0};
    const u32 s0 = x.ks[b] << 23, s1 = D == 256 ? x.ks[b] << 15 : s0;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const u32 scale = s < 4 ? s0 : s1;
      const bf16x8 k = as_bf16x8(decode<0>(x.k[b][s], scale), decode<1>(x.k[b][s], scale), decode<2>(x.k[b][s], scale), decode<3>(x.k[b][s], scale));
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t) sc[b][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, w.q[t][rb][s], sc[b][rb], 0, 0, 0);
    }
  }
  if (MASKED) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float s = poison ? __builtin_nanf("") : sc[b][rb][i];
          sc[b][rb][i] = sees[rb] >> (4 * b + i) & 1 ? s : -__builtin_inff();
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
  u32 p[TERMS][RB][4];
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
      for (int k = 0; k < TERMS; ++k) p[k][rb][h] = t[k];
    }
  }
  // scales of the eight keys; past the end of the sequence memory holds anything, and 0 times that has to be 0
  u32 vs[8];
  u32 s0 = x.vs[0], s1 = x.vs[1];
  if (MASKED) {
    const int n = there;  // of the lane's eight keys
    s0 = n >= 4 ? s0 : n <= 0 ? 0 : s0 & ((1u << (8 * n)) - 1);
    s1 = n >= 8 ? s1 : n <= 4 ? 0 : s1 & ((1u << (8 * (n - 4))) - 1);
  }
  vs[0] = scale_at<0>(s0); vs[1] = scale_at<1>(s0); vs[2] = scale_at<2>(s0); vs[3] = scale_at<3>(s0);
  vs[4] = scale_at<0>(s1); vs[5] = scale_at<1>(s1); vs[6] = scale_at<2>(s1); vs[7] = scale_at<3>(s1);
  auto product = [&](int f, u32 v0, u32 v1, u32 v2, u32 v3) {
    const bf16x8 v = as_bf16x8(v0, v1, v2, v3);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int t = TERMS - 1; t >= 0; --t)
        w.o[f][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, as_bf16x8(p[t][rb][0], p[t][rb][1], p[t][rb][2], p[t][rb][3]), w.o[f][rb], 0, 0, 0);
  };
  auto pairs = [&](auto byte, int f, const u32* words, u32 shift) {  // channels 2 byte, 2 byte + 1 of a dword column
    constexpr int BYTE = decltype(byte)::value;
    u32 y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = decode<BYTE>(words[j] >> shift, vs[j]);
    product(f, low_halves(y[0], y[1]), low_halves(y[2], y[3]), low_halves(y[4], y[5]), low_halves(y[6], y[7]));
    product(f + 1, high_halves(y[0], y[1]), high_halves(y[2], y[3]), high_halves(y[4], y[5]), high_halves(y[6], y[7]));
  };
  if constexpr (D == 64) {
    const u32 shift = (r & 1) * 16;
    pairs(std::integral_constant<int, 0>{}, 0, x.v, shift);
    pairs(std::integral_constant<int, 1>{}, 2, x.v, shift);
  } else {
#pragma unroll
    for (int h = 0; h < D / 128; ++h) {
      pairs(std::integral_constant<int, 0>{}, 8 * h, x.v + 8 * h, 0);
      pairs(std::integral_constant<int, 1>{}, 8 * h + 2, x.v + 8 * h, 0);
      pairs(std::integral_constant<int, 2>{}, 8 * h + 4, x.v + 8 * h, 0);
      pairs(std::integral_constant<int, 3>{}, 8 * h + 6, x.v + 8 * h, 0);
    }
  }
}

// Which of the keys first .. first + 7 (numbered from the first node on; committed ones are < 0) row `node` of n nodes sees.
__device__ __forceinline__ u32 seen(const AttnArgs& a, int b, int node, int n, int first) {
  u32 bits;
  if (a.mask) {
    const unsigned long long* row = a.mask + (static_cast<size_t>(b) * a.N + node) * a.words;
    auto word = [&](int w) { return w < 0 ? ~0ull : w < a.words ? row[w] : 0ull; };
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

// Where the results of a lane go: element [f][i] of row rb is channel (4g + i) * D/16 + f.
template <int D, int RB, typename T>
__device__ __forceinline__ void write_rows(const AttnArgs& a, int b, int head, int row0, int rb, int rows, const f32x4 (&o)[D / 16], float m, float l) {
  constexpr int C = D / 16;
  const int lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
  const int row = row0 + rb * 16 + r;
  if (row >= rows) return;
  const int node = row / a.group, h = head * a.group + row - node * a.group;
  const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
  T* at = static_cast<T*>(a.out) + b * a.out_request + node * a.out_node + h * a.out_head + g * (4 * C);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same<T, float>::value) {
#pragma unroll
      for (int f = 0; f < C; f += 4)
        *reinterpret_cast<f32x4*>(at + i * C + f) = f32x4{o[f][i] * inverse, o[f + 1][i] * inverse, o[f + 2][i] * inverse, o[f + 3][i] * inverse};
    } else if constexpr (C >= 8) {
#pragma unroll
      for (int f = 0; f < C; f += 8)
        *reinterpret_cast<u32x4*>(at + i * C + f) =
            u32x4{round_pair(o[f][i] * inverse, o[f + 1][i] * inverse), round_pair(o[f + 2][i] * inverse, o[f + 3][i] * inverse),
                  round_pair(o[f + 4][i] * inverse, o[f + 5][i] * inverse), round_pair(o[f + 6][i] * inverse, o[f + 7][i] * inverse)};
    } else {
      *reinterpret_cast<u32x2*>(at + i * C) = u32x2{round_pair(o[0][i] * inverse, o[1][i] * inverse), round_pair(o[2][i] * inverse, o[3][i] * inverse)};
    }
  }
  if (a.lse && g == 0)
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
template <int MODE, int RB> constexpr int rows_per_item = MODE == KEYS ? 16 * RB : 64 * RB;
template <int MODE> constexpr int unit_keys = MODE == KEYS ? 4 * kTile : kTile;

// One wave over keys [from, to) of an item; every `step`-th tile of 32 from `from` on.
template <int D, int RB, typename T>
__device__ __forceinline__ void run_keys(const AttnArgs& a, Wave<D, RB, T>& w, int b, int s, int head, int len, int n, int from, int to, int step) {
  const int lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
  const int end = len + n;
  // rows of a wave without a mask see nothing past their last node
  int last = end;
  if (!a.mask) {
    int node = -1;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) node = max(node, w.node[rb]);
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) node = max(node, __shfl_xor(node, d));
    last = min(end, len + 1 + __builtin_amdgcn_readfirstlane(node));
  }
  to = min(to, last);
  if (from >= to) return;
  const Reader<D> reader(a, s, head, end);
  Tile<D> x, next;
  int kpage = reader.page(from + (r >> 2) * 8), vpage = reader.page(from + g * 8);
  reader.load(from, kpage, vpage, next);
  int next_vpage = vpage;
  if (from + step < to) {
    kpage = reader.page(from + step + (r >> 2) * 8);
    vpage = reader.page(from + step + g * 8);
  }
  for (int t0 = from; t0 < to; t0 += step) {
    x = next;
    const bool poison = static_cast<u32>(next_vpage) >= static_cast<u32>(a.c.pages);
    if (t0 + step < to) {
      reader.load(t0 + step, kpage, vpage, next);
      next_vpage = vpage;
      if (t0 + 2 * step < to) {
        kpage = reader.page(t0 + 2 * step + (r >> 2) * 8);
        vpage = reader.page(t0 + 2 * step + g * 8);
      }
    }
    u32 sees[RB];
    if (t0 + kTile <= len && !__any(poison)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) sees[rb] = 0xFF;
      attend<D, RB, T, false>(w, x, a.scale_log2, sees, 8, false);
    } else {
      const int first = t0 + 8 * g;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) sees[rb] = w.node[rb] < 0 ? 0u : seen(a, b, w.node[rb], n, first - len);
      attend<D, RB, T, true>(w, x, a.scale_log2, sees, end - first, poison);
    }
  }
}

template <int D, int RB, typename T, int MODE>
__global__ void __launch_bounds__(kThreads) attention_kernel(AttnArgs a, u32 least) {
  constexpr int NF = D / 16, ROWS_ITEM = rows_per_item<MODE, RB>, UNIT = unit_keys<MODE>;
  using Dealt = Deal<ROWS_ITEM, UNIT>;
  __shared__ u32 sh_begin[MARS_KV_MAX_REQUESTS + 1];
  __shared__ float sh_m[MODE == KEYS ? 4 : 1][16 * RB], sh_l[MODE == KEYS ? 4 : 1][16 * RB];
  __shared__ __attribute__((aligned(16))) float sh_o[MODE == KEYS ? 2 : 1][MODE == KEYS ? RB * NF * 256 : 4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane % 16;

  if (a.n_new || a.seqs)  // (otherwise every request has N nodes)
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
      const Dealt d(a, b);
      if (d.n < a.N) clear_rows<T, D>(a, b, d.n);
    }
  deal_out<Dealt>(a, sh_begin);
  const u32 total = sh_begin[a.B], share = share_of(total, gridDim.x, least);
  // neighbours in the deal on the same die (block index mod 8)
  const u32 per_die = gridDim.x >> 3;
  const u32 group = (blockIdx.x & 7) * per_die + (blockIdx.x >> 3);
  const unsigned long long my_begin = static_cast<unsigned long long>(group) * share;
  if (my_begin >= total) return;
  const u32 unit0 = static_cast<u32>(my_begin), unit1 = static_cast<u32>(min(my_begin + share, static_cast<unsigned long long>(total)));

  Wave<D, RB, T> w;
  for (u32 u = unit0; u < unit1;) {
    const int b = request_of(sh_begin, a.B, u);
    const Dealt d(a, b);
    const u32 local = u - sh_begin[b];
    const int item = static_cast<int>(local / d.tiles), tile = static_cast<int>(local % d.tiles);
    const int tiles = static_cast<int>(min(static_cast<u32>(d.tiles - tile), unit1 - u));
    const bool whole = tile == 0 && tiles == d.tiles;
    const int blocks = d.items / a.c.heads;
    const int head = item / blocks, block = item % blocks, rows = d.n * a.group;
    const int row0 = block * ROWS_ITEM + (MODE == ROWS ? wave * 16 * RB : 0);
    const int s = sequence_of(a.c, a.seqs, b);
    w.start(a, b, head, row0, rows);
    const int from = tile * UNIT + (MODE == KEYS ? wave * kTile : 0), to = (tile + tiles) * UNIT;
    if (MODE == KEYS || row0 < rows) run_keys<D, RB, T>(a, w, b, s, head, d.len, d.n, from, to, UNIT);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) w.l[rb] = over_groups_sum(w.l[rb]);

    if (MODE == KEYS) {
      __syncthreads();  // (the piece before)
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
        f32x4* const sh = reinterpret_cast<f32x4*>(sh_o[wave & (half - 1)]) + lane;
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
          write_rows<D, RB, T>(a, b, head, row0, rb, rows, o, w.m[rb], w.l[rb]);
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
    u += tiles;
  }
}

// Joins the pieces of items that were dealt to several work-groups: one work-group for every place where the deal cuts one, of which the
// first of an item takes it; a wave per 16 rows.
template <int D, int RB, typename T, int MODE>
__global__ void __launch_bounds__(kThreads) merge_kernel(AttnArgs a, u32 groups, u32 least) {
  constexpr int NF = D / 16, ROWS_ITEM = rows_per_item<MODE, RB>, UNIT = unit_keys<MODE>;
  using Dealt = Deal<ROWS_ITEM, UNIT>;
  __shared__ u32 sh_begin[MARS_KV_MAX_REQUESTS + 1];
  deal_out<Dealt>(a, sh_begin);
  const u32 total = sh_begin[a.B], share = share_of(total, groups, least);
  const u32 cut = blockIdx.x + 1;
  const unsigned long long at = static_cast<unsigned long long>(cut) * share;
  if (at >= total) return;
  const int b = request_of(sh_begin, a.B, static_cast<u32>(at));
  const Dealt d(a, b);
  const u32 local = static_cast<u32>(at) - sh_begin[b];
  const int item = static_cast<int>(local / d.tiles);
  const u32 item0 = sh_begin[b] + static_cast<u32>(item) * d.tiles, item1 = item0 + d.tiles;
  if (item0 == at) return;                            // cut between two items
  const u32 first = item0 / share, last = (item1 - 1) / share;
  if (cut != first + 1) return;                       // an earlier cut's
  const int blocks = d.items / a.c.heads;
  const int head = item / blocks, block = item % blocks, rows = d.n * a.group;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane % 16;
  constexpr int STRIPS = MODE == ROWS ? 4 * RB : RB;   // of 16 rows
  for (int strip = blockIdx.y * 4 + wave; strip < STRIPS; strip += gridDim.y * 4) {
    const int part = MODE == ROWS ? strip / RB : 0, rb = MODE == ROWS ? strip % RB : strip;
    auto slot = [&](u32 group) {
      const u32 second = static_cast<unsigned long long>(group) * share >= item0 ? 0 : 1;
      return (static_cast<long>(group) * 2 + second) * (MODE == ROWS ? 4 : 1) + part;
    };
    float m = kFloor;
    for (u32 p = first; p <= last; ++p) m = fmaxf(m, Piece<D, RB>(a.partial, slot(p)).reference(rb * 16 + r));
    float l = 0.0f;
    f32x4 o[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) o[f] = f32x4{0, 0, 0, 0};
    for (u32 p = first; p <= last; ++p) {
      const Piece<D, RB> piece(a.partial, slot(p));
      const float weight = __builtin_amdgcn_exp2f(piece.reference(rb * 16 + r) - m);
      l += piece.sum(rb * 16 + r) * weight;
#pragma unroll
      for (int f = 0; f < NF; ++f) o[f] += piece.part(rb, f, lane) * weight;
    }
    write_rows<D, RB, T>(a, b, head, block * ROWS_ITEM + part * 16 * RB, rb, rows, o, m, l);
  }
}

}  // namespace kv
}  // namespace mars
