// C ABI of the paged 4-bit cache (see include/mars_cache.h): argument checks, workspace carving and kernel launches.  Nothing
// here allocates or synchronises.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/mars_cache.h"
#include "kv_attention.h"
#include "kv_format.h"
#include "kv_pages.h"
#include "kv_rows.h"

namespace mars {
namespace kv {

constexpr size_t kAlign = 256;
static size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
static int launched() { return hipGetLastError() == hipSuccess ? MARS_OK : MARS_ERR_HIP; }

enum { POOL = 1, TABLE = 2, LENS = 4, HELD = 8, REFS = 16 };

// The cache as the kernels see it, if it is one and has the tables that a call names.
static bool cache_ok(const mars_kv_cache* k, int needs, Cache* c) {
  if (!k || k->layers < 1 || k->pages < 1 || k->heads < 1 || k->sequences < 1 || k->width < 1) return false;
  if (mars_kv_head_bytes(k->dim, k->page) == 0) return false;
  if (((needs & POOL) && !k->pool) || ((needs & TABLE) && !k->page_table) || ((needs & LENS) && !k->lens) ||
      ((needs & HELD) && !k->held) || ((needs & REFS) && !k->refs))
    return false;
  if (reinterpret_cast<uintptr_t>(k->pool) % 16) return false;
  int log_page = 3;
  while ((1 << log_page) < k->page) ++log_page;
  const size_t blk = head_bytes(k->dim, k->page), page_bytes = blk * k->heads;
  if (page_bytes > (1u << 30) || k->pages > (1 << 30) || static_cast<long>(k->width) * k->page > (1l << 30)) return false;
  *c = Cache{static_cast<uint8_t*>(k->pool), k->page_table, k->lens, k->held, k->refs, page_bytes * k->pages,
             static_cast<u32>(page_bytes), static_cast<u32>(blk), k->layers, k->pages, k->heads, log_page, k->sequences, k->width};
  return true;
}
static bool batch_ok(int B, int N) { return B >= 1 && B <= MARS_KV_MAX_REQUESTS && N >= 1 && N <= (1 << 24); }
static bool dtype_ok(int dtype) { return dtype == MARS_F32 || dtype == MARS_BF16; }
static bool rows_ok(const mars_kv_rows* r, int dtype) {
  if (!r || !r->data || reinterpret_cast<uintptr_t>(r->data) % 16) return false;
  const int64_t step = dtype == MARS_F32 ? 4 : 8;
  return r->request % step == 0 && r->node % step == 0 && r->head % step == 0;
}
template <typename T> static Rows<T> rows_of(const mars_kv_rows* r) { return Rows<T>{static_cast<T*>(r->data), r->request, r->node, r->head}; }

// f(integral_constant<dim>).
template <typename F> static int by_dim(int dim, F f) {
  switch (dim) {
    case 64: return f(std::integral_constant<int, 64>{});
    case 128: return f(std::integral_constant<int, 128>{});
    default: return f(std::integral_constant<int, 256>{});
  }
}
// f(a value of the element type).
template <typename F> static int by_type(int dtype, F f) { return dtype == MARS_F32 ? f(float{}) : f(bf16_t{}); }

static int row_octets(int N) { return (N + 6) / 8 + 1; }  // octets that N positions can touch

// Work-groups of a commit, as long as each has as many layers as it takes at a time: 256 paths in 32 layers and 8 heads 45 us by about 4 096, 50 by
// 2 048; 32 paths 9.5 us by 512 of two layers, 11 by 1 024 of one.
constexpr int kCommitGroups = 4096;
// Pools of up to this many pages are searched for free ones by 256 threads (two steps of 4 096), larger ones by 1 024: two requests of 60 tokens, the free pages the last
// ones, 7.4 us by 256 threads and 7.6 by 1 024 in a pool of 4 000 pages, 8.0 and 7.1 in one of 16 000, 16 and 10 in one of 60 000 (106 and 55 us in one of 400 000: 128
// requests).
constexpr int kPlanFewPages = 8192;

// ---------------------------------------------------------------- attention: how the work is laid out
struct AttnPlan {
  int mode, rows;  // waves divide keys or rows; rows of a wave
  int waves;       // of a work-group
  int nodes;       // of a block of rows
  u32 groups;      // work-groups beside each other on the chip
  size_t bytes;    // of pieces
};
// Up to 32 rows of bf16 the waves divide the keys: 28 rows over 4 caches of 60 000 - 131 000 tokens take 110 us so, and 165 in blocks of 16.  Beyond, 32
// rows each, by 8 waves where their blocks hold no more rows than those of 4 (208 rows over long caches: 410 us, by 4 waves 480; 240 rows over 16 caches of 1 024 -
// 8 191: 117 and 125; a prompt of 2 048 nodes, 64 blocks of four waves: 241 and 260), else by 4 (100 rows: 76 us, by 8 waves 90; 288 rows: 159 and 167; 352: 164 and 173;
// 616, five blocks: 411 and 447).  With many blocks the odd one costs less than four waves do: 65 blocks, 2 049 or 2 080 nodes, take 272 us by 4 waves, and
// would take 255 by 8; the rule leaves that.
// In 32 bits the products take three times as long and 32 rows a third more registers: up to 80 rows 16 at a time are faster (48 rows: 47 us instead of 71, 80
// rows: 66 and 77; 120 rows: 97 and 84).
static AttnPlan attn_plan(int N, int group, int dim, int dtype, int page) {
  const long rows = static_cast<long>(N) * group;
  const bool f32 = dtype == MARS_F32;
  AttnPlan p;
  p.mode = (f32 ? group <= 16 && rows <= 80 : rows <= 32) ? KEYS : ROWS;
  p.rows = p.mode == KEYS && (f32 || rows <= 16) ? 16 : 32;
  const long four = (rows + kWaves * 32 - 1) / (kWaves * 32);  // blocks of four waves
  p.waves = p.mode == ROWS && four % 2 == 0 && !f32 && dim <= 128 ? 2 * kWaves : kWaves;
  p.groups = 256 * per_unit(dim, p.mode, p.waves, p.rows, f32, page >= kTile);
  p.nodes = (p.mode == ROWS ? p.waves * p.rows : p.rows) / group;
  // (a wave's piece: its rows' references and sums, and its results)
  const size_t piece = sizeof(float) * (2 * p.rows + static_cast<size_t>(p.rows) * dim);
  p.bytes = align_up(static_cast<size_t>(p.groups) * 2 * (p.mode == ROWS ? p.waves : 1) * piece);
  return p;
}
// Blocks of up to this many units (as far as the caller says) are not cut: their pieces would have to be joined, by a second kernel.  One token, 8
// heads, 1 021 tokens: 12 us, cut 15; 1 500: 15 and 12.5.  Where there are blocks enough for half the compute units, and each is a few rows of bf16
// (light), cutting wins less: 32 times one token over 1 900 - 2 000, 256 blocks: 19 us, cut 28; 8 times, 64 blocks: 18.6 and 17.7.
static int whole_units(bool light, long blocks) { return light && blocks >= 128 ? 16 : 8; }
// The same where the lengths decide (the second kernel runs in any case then), in units beyond an even share: 64 times one token over 5 000 67 us with 20, 82 with
// 12, 128 over 500 - 4 000 69 and 82; one over 1 500 18 and 13.  With more rows a unit takes longer: 8 trees of 240 rows over 1 000 - 1 900 72 us with 12, 46
// with 8, 46 with 0; 32 such trees 80, 80 and 94.
static u32 join_cost(bool light, long blocks) { return light && blocks >= 128 ? 20 : 8; }

// Units that a work-group takes at least: with two, pieces are half as many to join.  One token over 4 000: 14.7 us instead of 17.9, 8 over 1 500
// 14.9 and 19.0, 2 trees of 240 rows over 1 900 36 and 41; but 2 of 28 rows over 1 000 - 1 900 23.6 and 19.0, 2 of 7 in fp32 16.4 and 14.6, whose
// units take longer and whose pieces are small.  (Three: one token over 2 000 15.2 instead of 12.2.)
static u32 least_share(const AttnPlan& p, int dtype) { return p.mode == KEYS && (dtype == MARS_F32 || p.rows == 32) ? 1 : 2; }

// The most that a call deals out, as kv_deal.h counts it (in 32 bits): units of blocks or of pairs of blocks -- of an odd number, the last pair is as
// large as the others -- or two per item.
static double most_dealt(int B, int N, int heads, int nodes, bool masked, long most_len) {
  const long blocks = (static_cast<long>(N) + nodes - 1) / nodes;
  const bool paired = !masked && blocks > 1;
  const long per = paired ? (2 * most_len + (blocks + 1) * nodes + 2 * (kUnit - 1)) / kUnit : (most_len + N + kUnit - 1) / kUnit;
  return static_cast<double>(B) * heads * (paired ? (blocks + 1) / 2 : blocks) * (per > 2 ? per : 2);
}

template <typename W> static int launch_attention(u32 groups, const AttnArgs& a, hipStream_t stream) {
  static_assert(Piece<W>::kFloats == 2 * W::kRows + W::kRows * W::D, "as attn_plan counts them");
  if (a.c.log_page >= 5) hipLaunchKernelGGL((attention_kernel<W, true>), dim3(groups), dim3(W::kGroupWaves * kWave), 0, stream, a);
  else hipLaunchKernelGGL((attention_kernel<W, false>), dim3(groups), dim3(W::kGroupWaves * kWave), 0, stream, a);
  if (hipGetLastError() != hipSuccess) return MARS_ERR_HIP;
  if (a.whole) return MARS_OK;
  hipLaunchKernelGGL(merge_kernel<W>, dim3(groups - 1, W::kStrips), dim3(kThreads), 0, stream, a, groups);
  return launched();
}

static ReserveSpace reserve_space(char* ws, int pages, int B) {
  const size_t n = align_up(sizeof(int32_t) * B), all = align_up(sizeof(int32_t) * pages);
  ReserveSpace r;
  r.copy_src = reinterpret_cast<int32_t*>(ws);
  r.copy_dst = reinterpret_cast<int32_t*>(ws + n);
  r.copies = reinterpret_cast<int32_t*>(ws + 2 * n);
  r.found = reinterpret_cast<int32_t*>(ws + 2 * n + kAlign);
  r.former = reinterpret_cast<int32_t*>(ws + 2 * n + kAlign + all);
  r.asks = reinterpret_cast<int32_t*>(ws + 2 * n + kAlign + 2 * all);
  r.last = reinterpret_cast<int32_t*>(ws + 2 * n + kAlign + 3 * all);
  return r;
}
static u32 copy_groups(const Cache& c, long pairs) {
  const long items = pairs * c.layers * ((c.page_bytes + kCopyPart - 1) / kCopyPart);
  return static_cast<u32>(items < 2048 ? items : 2048);
}

}  // namespace kv
}  // namespace mars

using namespace mars::kv;

extern "C" {

size_t mars_kv_head_bytes(int dim, int page) {
  if ((dim != 64 && dim != 128 && dim != 256) || page < 8 || page > 256 || (page & (page - 1))) return 0;
  return head_bytes(dim, page);
}

int mars_kv_append(const mars_kv_cache* cache, int layer, const int32_t* seqs, const mars_kv_rows* k, const mars_kv_rows* v,
                   int dtype, const int32_t* n_new, int B, int N, int32_t* status, void* hip_stream) {
  Cache c;
  if (!batch_ok(B, N) || !cache_ok(cache, POOL | TABLE | LENS, &c) || layer < 0 || layer >= c.layers) return MARS_ERR_ARG;
  if (!dtype_ok(dtype)) return MARS_ERR_DTYPE;
  if (!rows_ok(k, dtype) || !rows_ok(v, dtype)) return MARS_ERR_ARG;
  const int octets = row_octets(N), per_group = 2048 / cache->dim;
  const long items = static_cast<long>(B) * octets * c.heads, groups = (items + per_group - 1) / per_group;
  if (groups > 0x7FFFFFFFl) return MARS_ERR_ARG;
  return by_dim(cache->dim, [&](auto dim) {
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      hipLaunchKernelGGL((append_kernel<decltype(dim)::value, T>), dim3(static_cast<u32>(groups)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), c,
                         c.layer_bytes * layer, seqs, rows_of<const T>(k), rows_of<const T>(v), n_new, B, N, octets, items, status);
      return launched();
    });
  });
}

int mars_kv_read(const mars_kv_cache* cache, int layer, const int32_t* seqs, const int32_t* first, const mars_kv_rows* k,
                 const mars_kv_rows* v, int dtype, int B, int N, void* hip_stream) {
  Cache c;
  if (!batch_ok(B, N) || !cache_ok(cache, POOL | TABLE, &c) || layer < 0 || layer >= c.layers) return MARS_ERR_ARG;
  if (!dtype_ok(dtype)) return MARS_ERR_DTYPE;
  if (!rows_ok(k, dtype) || !rows_ok(v, dtype)) return MARS_ERR_ARG;
  const int octets = row_octets(N), per_group = 2048 / cache->dim;
  const long items = static_cast<long>(B) * octets * c.heads, groups = (items + per_group - 1) / per_group;
  if (groups > 0x7FFFFFFFl) return MARS_ERR_ARG;
  return by_dim(cache->dim, [&](auto dim) {
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      hipLaunchKernelGGL((read_kernel<decltype(dim)::value, T>), dim3(static_cast<u32>(groups)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), c,
                         c.layer_bytes * layer, seqs, first, rows_of<T>(k), rows_of<T>(v), B, N, octets, items);
      return launched();
    });
  });
}

int mars_tree_mask(const int32_t* tree_parent, const int32_t* n_new, int B, int N, uint64_t* mask, int32_t* status, void* hip_stream) {
  if (!tree_parent || !mask || B < 1 || B > MARS_KV_MAX_REQUESTS || N < 1 || N > MARS_MAX_NODES) return MARS_ERR_ARG;
  hipLaunchKernelGGL(tree_mask_kernel, dim3(B), dim3(kMaskThreads), 0, static_cast<hipStream_t>(hip_stream), tree_parent, n_new, N,
                     reinterpret_cast<unsigned long long*>(mask), status);
  return launched();
}

static bool attention_sizes_ok(int B, int N, int q_heads, int heads, int dim) {
  return batch_ok(B, N) && heads >= 1 && q_heads >= heads && q_heads % heads == 0 && q_heads <= (1 << 16) && mars_kv_head_bytes(dim, 8) != 0 &&
         q_heads / heads <= 64 && static_cast<long>(N) * (q_heads / heads) <= (1l << 28);
}

size_t mars_kv_attention_workspace_bytes(int B, int N, int q_heads, int heads, int dim, int dtype) {
  if (!attention_sizes_ok(B, N, q_heads, heads, dim) || !dtype_ok(dtype)) return 0;
  return attn_plan(N, q_heads / heads, dim, dtype, kTile).bytes;  // (for pages of less it may be more than is wanted)
}

int mars_kv_attention(const mars_kv_cache* cache, int layer, const int32_t* seqs, const mars_kv_rows* q, int dtype, int q_heads,
                      const int32_t* n_new, const uint64_t* mask, float scale, int max_len, const mars_kv_rows* out, float* lse,
                      int B, int N, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Cache c;
  if (!batch_ok(B, N) || !cache_ok(cache, POOL | TABLE | LENS, &c) || layer < 0 || layer >= c.layers ||
      !attention_sizes_ok(B, N, q_heads, c.heads, cache->dim))
    return MARS_ERR_ARG;
  if (!dtype_ok(dtype)) return MARS_ERR_DTYPE;
  const float scale_log2 = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634);
  if (!rows_ok(q, dtype) || !rows_ok(out, dtype) || max_len < 0 || !(scale > 0.0f) || !std::isfinite(scale_log2) || (mask && N > MARS_MAX_NODES))
    return MARS_ERR_ARG;
  const AttnPlan p = attn_plan(N, q_heads / c.heads, cache->dim, dtype, cache->page);
  const long most_len = static_cast<long>(c.width) << c.log_page;
  if (most_dealt(B, N, c.heads, p.nodes, mask != nullptr, most_len) > 4.0e9) return MARS_ERR_ARG;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % kAlign || workspace_bytes < p.bytes) return MARS_ERR_WORKSPACE;
  AttnArgs a{};
  a.c = c;
  a.layer_offset = c.layer_bytes * layer;
  a.seqs = seqs;
  a.n_new = n_new;
  a.mask = reinterpret_cast<const unsigned long long*>(mask);
  a.q = q->data;
  a.q_request = q->request; a.q_node = q->node; a.q_head = q->head;
  a.out = out->data;
  a.out_request = out->request; a.out_node = out->node; a.out_head = out->head;
  a.lse = lse;
  a.partial = static_cast<float*>(workspace);
  a.scale_log2 = scale_log2;
  a.B = B; a.N = N; a.q_heads = q_heads; a.group = q_heads / c.heads; a.words = (N + 63) / 64;
  a.nodes = p.nodes;
  const long blocks = static_cast<long>(B) * c.heads * ((N + p.nodes - 1) / p.nodes);
  const double units = static_cast<double>(blocks) * ((most_len + N + 3 * kUnit) / kUnit);  // at most, about
  const bool light = p.mode == KEYS && dtype == MARS_BF16;
  a.whole = ((max_len && max_len < most_len ? max_len : most_len) + N + kUnit - 1) / kUnit <= whole_units(light, blocks);
  a.join_cost = join_cost(light, blocks);
  a.least_share = least_share(p, dtype);
  const double wanted = a.whole ? (blocks < (1 << 20) ? blocks : 1 << 20) : units < p.groups ? units : p.groups;
  const u32 groups = (static_cast<u32>(wanted) + 7) / 8 * 8;  // dealt out die by die
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  return by_dim(cache->dim, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    if (p.mode == KEYS) {
      if (dtype == MARS_F32) return launch_attention<Narrow<D, 1, float>>(groups, a, stream);
      return p.rows == 16 ? launch_attention<Narrow<D, 1, bf16_t>>(groups, a, stream) : launch_attention<Narrow<D, 2, bf16_t>>(groups, a, stream);
    }
    if (dtype == MARS_F32) return launch_attention<Wide<D, float, kWaves>>(groups, a, stream);
    if constexpr (D <= 128)
      if (p.waves > kWaves) return launch_attention<Wide<D, bf16_t, 2 * kWaves>>(groups, a, stream);
    return launch_attention<Wide<D, bf16_t, kWaves>>(groups, a, stream);
  });
}

int mars_kv_commit(const mars_kv_cache* cache, const int32_t* seqs, const int32_t* accept_len, const int32_t* path_idx, int B, int N,
                   int32_t* new_lens, int32_t* status, void* hip_stream) {
  Cache c;
  if (!batch_ok(B, N) || !cache_ok(cache, POOL | TABLE | LENS, &c) || !accept_len || !path_idx || !new_lens) return MARS_ERR_ARG;
  // layers per work-group
  const long quads = static_cast<long>(B) * ((c.heads + 3) / 4);
  const long even = (quads * c.layers + kCommitGroups - 1) / kCommitGroups, per_group = even < kCommitDeep ? kCommitDeep : even;
  const int layers = per_group < c.layers ? static_cast<int>(per_group) : c.layers;
  const long groups = quads * ((c.layers + layers - 1) / layers);
  if (groups > 0x7FFFFFFFl) return MARS_ERR_ARG;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  int32_t* apart = new_lens == c.lens ? nullptr : new_lens;
  const int rc = by_dim(cache->dim, [&](auto dim) {
    hipLaunchKernelGGL((commit_kernel<decltype(dim)::value>), dim3(static_cast<u32>(groups)), dim3(256), 0, stream, c, seqs, accept_len, path_idx, B, N,
                       layers, apart, status);
    return launched();
  });
  if (rc != MARS_OK || apart) return rc;
  hipLaunchKernelGGL(commit_lens_kernel, dim3((B + 3) / 4), dim3(256), 0, stream, c, seqs, accept_len, path_idx, B, N);
  return launched();
}

size_t mars_kv_reserve_workspace_bytes(int pages, int B) {
  if (pages < 1 || pages > (1 << 30) || B < 1 || B > MARS_KV_MAX_REQUESTS) return 0;
  return 2 * align_up(sizeof(int32_t) * B) + kAlign + 4 * align_up(sizeof(int32_t) * pages);
}

int mars_kv_reserve(const mars_kv_cache* cache, const int32_t* seqs, const int32_t* n_new, int B, int N, int32_t* status, void* workspace,
                    size_t workspace_bytes, void* hip_stream) {
  Cache c;
  if (!batch_ok(B, N) || !cache_ok(cache, POOL | TABLE | LENS | HELD | REFS, &c)) return MARS_ERR_ARG;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % kAlign || workspace_bytes < mars_kv_reserve_workspace_bytes(c.pages, B))
    return MARS_ERR_WORKSPACE;
  const ReserveSpace ws = reserve_space(static_cast<char*>(workspace), c.pages, B);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (B <= kPlanFew && c.pages <= kPlanFewPages)
    hipLaunchKernelGGL(reserve_kernel<kPlanFew>, dim3(1), dim3(kPlanFew), 0, stream, c, seqs, n_new, B, N, status, ws);
  else
    hipLaunchKernelGGL(reserve_kernel<kPlanMany>, dim3(1), dim3(kPlanMany), 0, stream, c, seqs, n_new, B, N, status, ws);
  if (hipGetLastError() != hipSuccess) return MARS_ERR_HIP;
  hipLaunchKernelGGL(copy_pages_kernel, dim3(copy_groups(c, B)), dim3(256), 0, stream, c, ws.copy_src, ws.copy_dst, ws.copies, 0);
  return launched();
}

int mars_kv_fork(const mars_kv_cache* cache, const int32_t* src, const int32_t* dst, int B, int32_t* status, void* hip_stream) {
  Cache c;
  if (!batch_ok(B, 1) || !cache_ok(cache, TABLE | LENS | HELD | REFS, &c) || !src || !dst) return MARS_ERR_ARG;
  hipLaunchKernelGGL(fork_kernel, dim3(B), dim3(256), 0, static_cast<hipStream_t>(hip_stream), c, src, dst, status);
  return launched();
}

int mars_kv_release(const mars_kv_cache* cache, const int32_t* seqs, int B, int32_t* status, void* hip_stream) {
  Cache c;
  if (!batch_ok(B, 1) || !cache_ok(cache, TABLE | LENS | HELD | REFS, &c)) return MARS_ERR_ARG;
  hipLaunchKernelGGL(release_kernel, dim3(B), dim3(256), 0, static_cast<hipStream_t>(hip_stream), c, seqs, status);
  return launched();
}

int mars_kv_copy_pages(const mars_kv_cache* cache, const int32_t* src, const int32_t* dst, int n, void* hip_stream) {
  Cache c;
  if (n < 1 || !cache_ok(cache, POOL, &c) || !src || !dst) return MARS_ERR_ARG;
  hipLaunchKernelGGL(copy_pages_kernel, dim3(copy_groups(c, n)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), c, src, dst, nullptr, n);
  return launched();
}

}  // extern "C"
