// Rows into the cache, out of it, and from one place in it to another (include/mars_cache.h): all bound by memory, or, for a step's
// few rows, by the latency of their chain of loads (length, page, row).
#pragma once

#include "kv_format.h"

namespace mars {
namespace kv {

template <typename T> struct Rows {
  T* data;
  long request, node, head;  // strides in elements
  __device__ __forceinline__ T* at(long b, long i, long h) const { return data + b * request + i * node + h * head; }
};

// A token's status within its request is written once, by the work-group of the request's first item.
__device__ __forceinline__ void report(int32_t* status, int b, int value) {
  if (status) status[b] = value;
}

// ---------------------------------------------------------------- append
// An item is eight positions beside each other (an octet: the unit of the values' layout) of a head; D/8 lanes take eight channels
// each and go through the octet's tokens, all of whose loads are under way before the first is used.  So a value's codes leave as
// 32 contiguous bytes per lane where the whole octet is new, and no lane ever reads what another one writes.
// 8 prompts of up to 8 192 tokens (8 heads of 128 channels): bf16, 198 MB read and written, 65 us, 3.0 TB/s, waiting for memory; fp32, 355 MB, 113 us, 3.1 TB/s (three waves per
// SIMD instead of five).  16 trees of 60 nodes 6.2 us.  The status is found by one lane, page after page: 1 025 pages of 8 tokens 100 us, 129 of 64 tokens 5.
template <int D, typename T>
__global__ void __launch_bounds__(256) append_kernel(Cache c, size_t layer_offset, const int32_t* __restrict__ seqs, Rows<const T> k,
                                                     Rows<const T> v, const int32_t* __restrict__ n_new, int B, int N, int octets,
                                                     long items, int32_t* __restrict__ status) {
  constexpr int LANES = D / 8, PER_GROUP = 256 / LANES;
  const int lane = threadIdx.x % LANES;
  const long item = static_cast<long>(blockIdx.x) * PER_GROUP + threadIdx.x / LANES;
  const bool live = item < items;
  const int h = live ? static_cast<int>(item % c.heads) : 0;
  const long bo = live ? item / c.heads : 0;
  const int o = static_cast<int>(bo % octets), b = static_cast<int>(bo / octets);
  const int s = sequence_of(c, seqs, b);
  const int n = n_new ? min(max(n_new[b], 0), N) : N;
  if (live && s < 0) {
    if (h == 0 && o == 0 && lane == 0) report(status, b, MARS_KV_BAD_SEQUENCE);
  }
  const int len = s >= 0 ? c.lens[s] : 0;
  if (live && s >= 0 && status && h == 0 && o == 0 && lane == 0) {
    int missing = len < 0;
    for (long i = len >> c.log_page; n > 0 && i <= ((static_cast<long>(len) + n - 1) >> c.log_page); ++i)
      missing |= i >= c.width || static_cast<u32>(c.page_table[static_cast<size_t>(s) * c.width + i]) >= static_cast<u32>(c.pages);
    status[b] = missing ? MARS_KV_NO_PAGES : MARS_KV_OK;
  }
  const int start = (len & ~7) + 8 * o;  // first position of the octet
  const int page = live && s >= 0 && len >= 0 ? page_of(c, s, start) : -1;
  // the octet's tokens among the new ones: positions start + from .. start + to - 1
  const int from = max(len - start, 0), to = page < 0 ? 0 : min(len + n - start, 8);

  Raw<T> kr[8], vr[8];  // (widened one by one: twice the registers otherwise, and three waves per SIMD instead of five with bf16)
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (j >= from && j < to) {
      kr[j] = load_raw(k.at(b, start + j - len, h) + lane * 8);
      vr[j] = load_raw(v.at(b, start + j - len, h) + lane * 8);
    }
  }
  const u32 t0 = start & ((1 << c.log_page) - 1);
  uint8_t* const base = head_of(c, layer_offset, max(page, 0), h);
  const int first_lane = (threadIdx.x % kWave) / LANES * LANES;
  const unsigned long long mine = (LANES == 64 ? ~0ull : (1ull << (LANES % 64)) - 1) << first_lane;
  u32 vw[8], vs[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool here = j >= from && j < to;
    const Eight kx = widen(kr[j]), vx = widen(vr[j]);
    const u32 kt = here ? top_bits(kx) : 0, vt = here ? top_bits(vx) : 0;
    const bool bad = (__ballot(max(kt, vt) >= 0x7F800000u) & mine) != 0;
    const u32 kb = scale_byte(block_top(kt)), vb = scale_byte(block_top(vt));
    vw[j] = vs[j] = 0;
    if (here) {
      *reinterpret_cast<u32*>(base + Place<D>::key(t0 + j) + lane * 4) = bad ? 0 : encode(kx, kb);
      if (lane % 4 == 0) base[Place<D>::key_scale(c.log_page, t0 + j) + lane / 4] = static_cast<uint8_t>(bad ? kNanScale : kb);
      vw[j] = bad ? 0 : encode(vx, vb);
      vs[j] = bad ? kLeastScale : vb;
    }
  }
  uint8_t* const vat = base + Place<D>::value(c.log_page, t0) + lane * 32;
  uint8_t* const sat = base + Place<D>::value_scale(c.log_page, t0) + lane / 4 * 8;
  if (from == 0 && to == 8) {
    reinterpret_cast<u32x4*>(vat)[0] = u32x4{vw[0], vw[1], vw[2], vw[3]};
    reinterpret_cast<u32x4*>(vat)[1] = u32x4{vw[4], vw[5], vw[6], vw[7]};
    if (lane % 4 == 0)
      *reinterpret_cast<u32x2*>(sat) = u32x2{vs[0] | vs[1] << 8 | vs[2] << 16 | vs[3] << 24, vs[4] | vs[5] << 8 | vs[6] << 16 | vs[7] << 24};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= from && j < to) {
        reinterpret_cast<u32*>(vat)[j] = vw[j];
        if (lane % 4 == 0) sat[j] = static_cast<uint8_t>(vs[j]);
      }
    }
  }
}

// ---------------------------------------------------------------- read
__device__ __forceinline__ void store_eight(float* p, const u32 (&w)[4]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u), __uint_as_float(w[1] << 16),
                                       __uint_as_float(w[1] & 0xFFFF0000u)};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{__uint_as_float(w[2] << 16), __uint_as_float(w[2] & 0xFFFF0000u),
                                           __uint_as_float(w[3] << 16), __uint_as_float(w[3] & 0xFFFF0000u)};
}
__device__ __forceinline__ void store_eight(bf16_t* p, const u32 (&w)[4]) { *reinterpret_cast<u32x4*>(p) = u32x4{w[0], w[1], w[2], w[3]}; }
__device__ __forceinline__ void decode_eight(u32 codes, u32 byte, u32 (&w)[4]) {
  const u32 scale = byte << 23;
  w[0] = decode<0>(codes, scale);
  w[1] = decode<1>(codes, scale);
  w[2] = decode<2>(codes, scale);
  w[3] = decode<3>(codes, scale);
}

// The items of append, the other way round.  Positions without a page are zero.  The same prompts, all N rows: bf16, 42 MB in and 268 out, 54 us, 5.7 TB/s, bound by
// the way out (a large copy reaches 4.9 in both directions together); fp32, 579 MB, 143 us.
template <int D, typename T>
__global__ void __launch_bounds__(256) read_kernel(Cache c, size_t layer_offset, const int32_t* __restrict__ seqs,
                                                   const int32_t* __restrict__ first, Rows<T> k, Rows<T> v, int B, int N, int octets,
                                                   long items) {
  constexpr int LANES = D / 8, PER_GROUP = 256 / LANES;
  const int lane = threadIdx.x % LANES;
  const long item = static_cast<long>(blockIdx.x) * PER_GROUP + threadIdx.x / LANES;
  if (item >= items) return;
  const int h = static_cast<int>(item % c.heads);
  const long bo = item / c.heads;
  const int o = static_cast<int>(bo % octets), b = static_cast<int>(bo / octets);
  const int s = sequence_of(c, seqs, b);
  const int begin = first ? first[b] : 0;
  const long start = (static_cast<long>(begin) & ~7l) + 8 * o;
  int page = -1;
  if (s >= 0 && start >= 0 && start <= 0x7FFFFFFFl) {
    page = page_of(c, s, static_cast<int>(start));
    if (c.held && (start >> c.log_page) >= c.held[s]) page = -1;
  }
  const int from = static_cast<int>(max(begin - start, 0l)), to = static_cast<int>(min(begin + static_cast<long>(N) - start, 8l));
  const u32 t0 = static_cast<u32>(start) & ((1u << c.log_page) - 1);
  const uint8_t* const base = head_of(c, layer_offset, max(page, 0), h);
  u32 kw[8], vw[8], ks[8], vs[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    kw[j] = vw[j] = 0;
    ks[j] = vs[j] = kLeastScale;
    if (page >= 0 && j >= from && j < to) {
      kw[j] = *reinterpret_cast<const u32*>(base + Place<D>::key(t0 + j) + lane * 4);
      vw[j] = *reinterpret_cast<const u32*>(base + Place<D>::value(c.log_page, t0 + j) + lane * 32);
      ks[j] = base[Place<D>::key_scale(c.log_page, t0 + j) + lane / 4];
      vs[j] = base[Place<D>::value_scale(c.log_page, t0 + j) + lane / 4 * 8];
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (j >= from && j < to) {
      u32 w[4];
      decode_eight(kw[j], ks[j], w);
      store_eight(k.at(b, start + j - begin, h) + lane * 8, w);
      decode_eight(vw[j], ks[j] == kNanScale ? kNanScale : vs[j], w);
      store_eight(v.at(b, start + j - begin, h) + lane * 8, w);
    }
  }
}

// ---------------------------------------------------------------- commit
// A wave takes the accepted rows of a request in one (layer, head), a lane a piece of a row (a dword of codes, a byte of scales) at every
// position.  The i-th row comes from path[i] and goes to 1 + i behind the committed tokens; path increases, so path[i] > i, and a row
// is written only where rows up to it have been read: batches of eight loads, then eight stores, in order, are safe in place.
struct Path {
  int seq, len, n;  // n: rows that move; 0 also where the request is refused
  int status;
};
// The request's path, checked by the whole wave (lane l looks at entries l, l + 64, ...).
__device__ __forceinline__ Path check_path(const Cache& c, const int32_t* seqs, const int32_t* accept_len, const int32_t* path_idx, int b, int N) {
  Path p;
  p.seq = sequence_of(c, seqs, b);
  p.len = p.seq >= 0 ? c.lens[p.seq] : 0;
  p.n = accept_len[b];
  p.status = MARS_KV_OK;
  bool bad = p.n < 0 || p.n >= N, missing = p.seq >= 0 && page_of(c, p.seq, p.len) < 0;  // (the root's row; len < 0 has no page either)
  if (p.seq >= 0 && !bad) {
    const int32_t* path = path_idx + static_cast<size_t>(b) * N;
    for (int i = threadIdx.x % kWave; i < p.n; i += kWave) {
      const int node = path[i], before = i ? path[i - 1] : 0;
      const bool in = node > before && node < N;
      bad |= !in;
      if (in) missing |= page_of(c, p.seq, p.len + node) < 0 || page_of(c, p.seq, p.len + 1 + i) < 0;
    }
  }
  if (p.seq < 0) p.status = MARS_KV_BAD_SEQUENCE;
  else if (__any(bad)) p.status = MARS_KV_BAD_PATH;
  else if (__any(missing)) p.status = MARS_KV_NO_PAGES;
  if (p.status != MARS_KV_OK) p.n = 0;
  return p;
}
// Where dword `i` of a token's codes (keys', then values'), and byte `i` of its scales, lie in a head's part of its page.
template <int D> __device__ __forceinline__ u32 dword_at(u32 log_page, u32 t, int i) {
  return i < D / 8 ? Place<D>::key(t) + i * 4 : Place<D>::value(log_page, t) + (i - D / 8) * 32;
}
template <int D> __device__ __forceinline__ u32 scale_byte_at(u32 log_page, u32 t, int i) {
  return i < D / 32 ? Place<D>::key_scale(log_page, t) + i : Place<D>::value_scale(log_page, t) + (i - D / 32) * 8;
}
// The path is looked at once for `per_group` layers: a wave's chain of loads (length, path, pages) costs as much as a dozen rows, and with a work-group per layer
// 256 paths in 32 layers took 8 rounds of it (67 us; now 45 from memory and 35 from the memory-side cache, some 160 MB in pieces of four bytes of the values and
// 64 of the keys, a third of which have to move).  16 paths in 32 layers: 7 us, latency.  Two layers at a time: with four, the registers leave room for four waves
// per SIMD (64 paths 16 us instead of 13.5, of 256 channels 24 instead of 14).
constexpr int kCommitDeep = 2;
template <int D>
__global__ void __launch_bounds__(256) commit_kernel(Cache c, const int32_t* __restrict__ seqs, const int32_t* __restrict__ accept_len,
                                                     const int32_t* __restrict__ path_idx, int B, int N, int per_group,
                                                     int32_t* __restrict__ new_lens, int32_t* __restrict__ status) {
  constexpr int BATCH = 8, DEEP = kCommitDeep;     // rows, and layers of them, on their way at a time
  constexpr int WORDS = D / 4, BYTES = D / 16;     // of a row
  constexpr int WORD_OPS = BATCH * WORDS / kWave, BYTE_OPS = (BATCH * BYTES + kWave - 1) / kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int quads = (c.heads + 3) / 4, parts = (c.layers + per_group - 1) / per_group;
  const int b = blockIdx.x / (parts * quads), rest = blockIdx.x % (parts * quads);
  const int layer0 = rest / quads * per_group, layer1 = min(layer0 + per_group, c.layers), h = rest % quads * 4 + wave;
  const Path p = check_path(c, seqs, accept_len, path_idx, b, N);
  if (rest == 0 && threadIdx.x == 0) {
    report(status, b, p.status);
    if (new_lens && p.seq >= 0) new_lens[p.seq] = p.status == MARS_KV_OK ? p.len + 1 + p.n : p.len;
  }
  if (h >= c.heads) return;
  const int32_t* path = path_idx + static_cast<size_t>(b) * N;
  const u32 in_page = (1u << c.log_page) - 1;
  for (int i0 = 0; i0 < p.n; i0 += BATCH) {
    // lane i < 8: source of row i0 + i, lane 8 + i: its target; -1: no row, or it stays where it is (a chain's)
    int at = -1, page = -1;
    const int i = i0 + lane % BATCH;
    if (lane < 2 * BATCH && i < p.n) {
      const int node = path[i];
      if (node != 1 + i) {
        at = p.len + (lane < BATCH ? node : 1 + i);
        page = page_of(c, p.seq, at);
      }
    }
    // the rows that move, beside each other
    const u32 moves = static_cast<u32>(__ballot(lane < BATCH && page >= 0));
    if (!moves) continue;
    const int rows = __popc(moves);
    auto place = [&](int q, bool source, auto where) -> long {  // offset of the q-th row's piece; -1: no such row
      u32 rest = moves;
      for (int k = 0; k < BATCH - 1; ++k)
        if (k < q) rest &= rest - 1;
      const int j = (q < rows ? __ffs(rest) - 1 : 0) + (source ? 0 : BATCH);
      const u32 of = __shfl(page, j), t = __shfl(at, j);  // (by all lanes: these are the ones that are read)
      return q < rows ? static_cast<long>(of) * c.page_bytes + static_cast<long>(h) * c.blk + where(t & in_page) : -1;
    };
    long word_from[WORD_OPS], word_to[WORD_OPS], byte_from[BYTE_OPS], byte_to[BYTE_OPS];
#pragma unroll
    for (int o = 0; o < WORD_OPS; ++o) {
      const int piece = o * kWave + lane, q = piece / WORDS;
      auto where = [&](u32 t) { return dword_at<D>(c.log_page, t, piece % WORDS); };
      word_from[o] = place(q, true, where);
      word_to[o] = place(q, false, where);
    }
#pragma unroll
    for (int o = 0; o < BYTE_OPS; ++o) {
      const int piece = o * kWave + lane, q = piece / BYTES;
      auto where = [&](u32 t) { return scale_byte_at<D>(c.log_page, t, piece % BYTES); };
      byte_from[o] = place(q, true, where);
      byte_to[o] = place(q, false, where);
    }
    for (int layer = layer0; layer < layer1; layer += DEEP) {
      uint8_t* const base = c.pool + static_cast<size_t>(layer) * c.layer_bytes;
      u32 x[DEEP][WORD_OPS], y[DEEP][BYTE_OPS];
#pragma unroll
      for (int d = 0; d < DEEP; ++d) {
        if (layer + d >= layer1) break;
#pragma unroll
        for (int o = 0; o < WORD_OPS; ++o)
          if (o * kWave / WORDS < rows && word_from[o] >= 0) x[d][o] = *reinterpret_cast<const u32*>(base + d * c.layer_bytes + word_from[o]);
#pragma unroll
        for (int o = 0; o < BYTE_OPS; ++o)
          if (byte_from[o] >= 0) y[d][o] = base[d * c.layer_bytes + byte_from[o]];
      }
#pragma unroll
      for (int d = 0; d < DEEP; ++d) {
        if (layer + d >= layer1) break;
#pragma unroll
        for (int o = 0; o < WORD_OPS; ++o)
          if (o * kWave / WORDS < rows && word_to[o] >= 0) *reinterpret_cast<u32*>(base + d * c.layer_bytes + word_to[o]) = x[d][o];
#pragma unroll
        for (int o = 0; o < BYTE_OPS; ++o)
          if (byte_to[o] >= 0) base[d * c.layer_bytes + byte_to[o]] = static_cast<uint8_t>(y[d][o]);
      }
    }
  }
}
// new_lens where it is lens itself: behind the kernel that reads it.  A wave per request.
__global__ void __launch_bounds__(256) commit_lens_kernel(Cache c, const int32_t* __restrict__ seqs, const int32_t* __restrict__ accept_len,
                                                          const int32_t* __restrict__ path_idx, int B, int N) {
  const int b = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (b >= B) return;
  const Path p = check_path(c, seqs, accept_len, path_idx, b, N);
  if (threadIdx.x % kWave == 0 && p.seq >= 0 && p.status == MARS_KV_OK) c.lens[p.seq] = p.len + 1 + p.n;
}

// ---------------------------------------------------------------- pages
// Whole pages from src to dst in all layers: work-groups go through (pair, layer, part of 16 KB).  `pairs`: how many there are,
// on the device (those of a reserve), or NULL: n.  120 pages of 32 layers, 535 MB read and written: 98 us, 5.4 TB/s.
constexpr int kCopyPart = 16384;
__global__ void __launch_bounds__(256) copy_pages_kernel(Cache c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                         const int32_t* __restrict__ pairs, int n) {
  const int parts = (c.page_bytes + kCopyPart - 1) / kCopyPart;
  const long items = static_cast<long>(pairs ? *pairs : n) * c.layers * parts;
  for (long item = blockIdx.x; item < items; item += gridDim.x) {
    const int part = static_cast<int>(item % parts), layer = static_cast<int>(item / parts % c.layers);
    const long i = item / parts / c.layers;
    const int from = src[i], to = dst[i];
    if (static_cast<u32>(from) >= static_cast<u32>(c.pages) || static_cast<u32>(to) >= static_cast<u32>(c.pages)) continue;
    const u32 begin = part * kCopyPart, end = min(begin + kCopyPart, c.page_bytes);
    const uint8_t* a = head_of(c, static_cast<size_t>(layer) * c.layer_bytes, from, 0);
    uint8_t* z = head_of(c, static_cast<size_t>(layer) * c.layer_bytes, to, 0);
    u32x4 x[kCopyPart / 4096];
#pragma unroll
    for (int j = 0; j < kCopyPart / 4096; ++j) {
      const u32 at = begin + j * 4096 + threadIdx.x * 16;
      if (at < end) x[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a + at));
    }
#pragma unroll
    for (int j = 0; j < kCopyPart / 4096; ++j) {
      const u32 at = begin + j * 4096 + threadIdx.x * 16;
      if (at < end) *reinterpret_cast<u32x4*>(z + at) = x[j];
    }
  }
}

}  // namespace kv
}  // namespace mars
