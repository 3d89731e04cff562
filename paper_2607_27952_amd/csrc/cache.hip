// Pages of a cache: whole pages copied, and a prompt's cache compacted to its
// text and kept visual tokens (Sec. 3.4, Eq. 12 on the cache). Both move rows
// of Dh elements, 16 bytes a thread, between pages of one pool; the host has
// checked that no row written is one that is read. The memory bounds both.
//
// Copy: a piece a thread, many blocks, one pool after the other. 1024 pages of
// 64 tokens and 8 heads in 2 layers, 1.07 GB moved, take 179 us (6.0 TB/s; four
// pieces a thread 207); 2000 pages of 16 tokens and 4 heads in 4 layers 102
// (109 with the layers of a page one after the other).
// Prune keeps single rows of 128 to 512 bytes: 64 sequences of 640 tokens to
// 128, 2 layers of 32 heads, 537 MB moved, 107 us (5.0 TB/s).
#include <algorithm>

#include "last_internal.h"

namespace {

using last::CopyArgs;
using last::PruneArgs;

constexpr int kRowsPrune = 32;   // most new tokens of a block
constexpr int kItems = 4;        // 16-byte pieces of a thread
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Piece i of a tile of rows of `1 << lc` 16-byte pieces, `inner` of them beside
// each other: its place in its row, and the row's two indices.
struct Cell {
  int c, inner, outer;
};
__device__ __forceinline__ Cell cell(uint32_t i, int lc, uint32_t inner) {
  const uint32_t row = i >> lc, o = row / inner;
  return Cell{(int)(i & ((1u << lc) - 1)), (int)(row - o * inner), (int)o};
}

__global__ __launch_bounds__(256) void k_cache_copy(CopyArgs a) {
  int64_t b = blockIdx.x;
  const int chunk = (int)(b % a.chunks);
  b /= a.chunks;
  const int64_t i = b % a.n;   // one pool after the other: they share no translations
  b /= a.n;
  const int kv = (int)(b & 1), g = (int)(b >> 1);
  const int32_t from = a.src[i], to = a.dst[i];
  if ((uint32_t)from >= (uint32_t)a.n_pages || (uint32_t)to >= (uint32_t)a.n_pages) return;
  u32x4 *base = (u32x4 *)(kv ? a.v : a.k) + g * a.layer_stride;
  const u32x4 *s = base + from * a.page_stride;
  u32x4 *d = base + to * a.page_stride;
  const uint32_t p = chunk * 256 + threadIdx.x;
  if (p >= (uint32_t)a.pieces) return;
  const Cell e = cell(p, a.lc, a.inner);
  const int64_t at = e.c + e.inner * a.inner_stride + e.outer * a.outer_stride;
  d[at] = s[at];
}

// Where token t of a sequence lies, in pieces from its layer's start; -1 where
// the table names no page of the cache.
__device__ __forceinline__ int64_t place(const PruneArgs &a, const int32_t *row, int t) {
  const int32_t page = row[t >> a.lg_page];
  if ((uint32_t)page >= (uint32_t)a.n_pages) return -1;
  return page * a.page_stride + (t & ((1 << a.lg_page) - 1)) * a.token_stride;
}

__global__ __launch_bounds__(256) void k_cache_prune(PruneArgs a) {
  __shared__ int64_t from[kRowsPrune], to[kRowsPrune];
  int64_t b = blockIdx.x;
  const int tile = (int)(b % a.tiles);
  b /= a.tiles;
  const int pools = 2 * a.G, sets = (pools - 1) / a.span + 1;
  const int first = (int)(b % sets) * a.span, last = min(pools, first + a.span);   // pools: keys and values of a layer
  const int r = (int)(b / sets);
  const int len = a.lens[r], vis = a.vis_start[r];
  const int n = a.cu_vis[r + 1] - a.cu_vis[r], k = a.cu_keep[r + 1] - a.cu_keep[r];
  const int m = max(0, min(len - n + k, a.max_new));
  if (a.new_lens && tile == 0 && first == 0 && threadIdx.x == 0) a.new_lens[r] = m;
  const int i0 = tile * a.rows;
  if (i0 >= m) return;
  if ((int)threadIdx.x < a.rows) {
    const int i = i0 + threadIdx.x;
    int64_t s = -1, d = -1;   // no source: zeros; no target: nothing
    if (i < m) {
      int old = i;
      if (i >= vis + k) old = i - k + n;
      else if (i >= vis) {
        const int x = a.kept[a.cu_keep[r] + i - vis];
        old = x >= 0 && x < n ? vis + x : -1;
      }
      const int32_t *st = a.src + (int64_t)r * a.src_pages, *dt = a.dst + (int64_t)r * a.dst_pages;
      if (old >= 0 && old < len && old < a.max_old) s = place(a, st, old);
      d = place(a, dt, i);
      if (s == d) d = -1;   // a shared page before the visual span
    }
    from[threadIdx.x] = s;
    to[threadIdx.x] = d;
  }
  __syncthreads();
  // Rows in the order they lie in: heads of a token, or tokens of a head. All
  // of a thread's loads are issued before its first store: loads and stores
  // count together, so a load behind a store would wait for that too.
  const uint32_t inner = a.heads_inner ? a.Hkv : a.rows;
  const uint32_t pieces = ((uint32_t)a.Hkv * a.rows) << a.lc, total = pieces * (last - first);
  for (uint32_t u0 = 0; u0 < total; u0 += 256 * kItems) {
    u32x4 x[kItems];
    u32x4 *dst[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
      dst[j] = nullptr;
      if (u0 + j * 256 >= total) continue;   // the whole block has no more
      const uint32_t u = min(u0 + j * 256 + threadIdx.x, total - 1), o = u / pieces;
      const Cell e = cell(u - o * pieces, a.lc, inner);
      const int head = a.heads_inner ? e.inner : e.outer, t = a.heads_inner ? e.outer : e.inner, c = first + o;
      u32x4 *base = (u32x4 *)(c & 1 ? a.v : a.k) + (c >> 1) * a.layer_stride + e.c + head * a.head_stride;
      const int64_t f = from[t], d = to[t];
      if (d >= 0 && u0 + j * 256 + threadIdx.x < total) dst[j] = base + d;
      x[j] = u32x4{};
      if (dst[j] && f >= 0) x[j] = base[f];
    }
#pragma unroll
    for (int j = 0; j < kItems; ++j)
      if (dst[j]) __builtin_nontemporal_store(x[j], dst[j]);
  }
}

}  // namespace

namespace last {

int64_t copy_blocks(CopyArgs *a) {
  a->chunks = (a->pieces + 255) / 256;
  return (int64_t)a->n * a->G * 2 * a->chunks;
}

hipError_t launch_cache_copy(const CopyArgs &a, int64_t blocks, hipStream_t s) {
  launch_begin("cache_copy", s);
  hipLaunchKernelGGL(k_cache_copy, dim3((unsigned)blocks), dim3(256), 0, s, a);
  return launch_end(s);
}

// A block moves as many tokens as give its threads a piece each (2 at least,
// for 32 heads: 107 us against 112 with 4 and 110 with 1), in so many layers'
// keys and values that a thread has up to kItems pieces, if that leaves 4
// blocks a compute unit: what it looks up (where each token comes from and
// goes to) then serves all of them. Eight sequences of 16384 visual tokens to
// 1024, 4 layers of 4 heads: 32 us, one pool a block 40; 32 sequences of 288 to
// 16384 to a ninth, 4 layers of 2 heads: 26, one pool a block 53.
// Tiles are counted by the longest sequence, whose blocks the shorter ones
// leave at once. Where a launch does not hold so many, a block takes every pool
// (as many as 32 bits count the pieces of), then the most tokens.
int64_t prune_blocks(PruneArgs *a) {
  const int64_t pools = 2 * (int64_t)a->G;
  auto set_rows = [a](int rows) {
    a->rows = rows;
    a->tiles = std::max(1, (a->max_new + rows - 1) / rows);
  };
  auto pieces = [a] { return ((int64_t)a->Hkv * a->rows) << a->lc; };
  auto set_span = [a, pools](int64_t span) { a->span = (int32_t)std::max<int64_t>(1, std::min(pools, span)); };
  auto blocks = [a, pools] { return (int64_t)a->R * a->tiles * ((pools + a->span - 1) / a->span); };
  set_rows(std::max(2, std::min(kRowsPrune, 256 / std::min(256, a->Hkv << a->lc))));
  set_span(std::min(256 * kItems / pieces(), (int64_t)a->R * pools * a->tiles / (4 * device_cus())));
  if (blocks() >= kMaxBlocks) set_span(((int64_t)1 << 31) / pieces());
  if (blocks() >= kMaxBlocks) {
    set_rows(kRowsPrune);
    set_span(((int64_t)1 << 31) / pieces());
  }
  return blocks();
}

hipError_t launch_cache_prune(const PruneArgs &a, int64_t blocks, hipStream_t s) {
  launch_begin("cache_prune", s);
  hipLaunchKernelGGL(k_cache_prune, dim3((unsigned)blocks), dim3(256), 0, s, a);
  return launch_end(s);
}

}  // namespace last
