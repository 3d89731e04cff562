// Pages of a cache: whole pages copied, and a prompt's cache compacted to its
// text and kept visual tokens (Sec. 3.4, Eq. 12 on the cache). Both move rows
// of Dh elements, 16 bytes a thread, between pages of one pool; the host has
// checked that no row written is one that is read.
#include <algorithm>

#include "last_internal.h"

namespace {

using last::CopyArgs;
using last::PruneArgs;

constexpr int kRowsPrune = 16;   // new tokens of a block
constexpr int kItems = 4;        // 16-byte pieces a thread has in flight

// Piece i of a tile of `inner` x `outer` rows of `1 << lc` pieces, as its
// offset in 16-byte pieces; inner rows are inner_stride pieces apart.
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
  const int kv = (int)(b & 1);
  b >>= 1;
  const int g = (int)(b % a.G);
  const int64_t i = b / a.G;
  const int32_t from = a.src[i], to = a.dst[i];
  if ((uint32_t)from >= (uint32_t)a.n_pages || (uint32_t)to >= (uint32_t)a.n_pages) return;
  uint4 *base = (uint4 *)(kv ? a.v : a.k) + g * a.layer_stride;
  const uint4 *s = base + from * a.page_stride;
  uint4 *d = base + to * a.page_stride;
  const uint32_t first = chunk * (256 * kItems) + threadIdx.x;
  uint4 x[kItems];
  int64_t at[kItems];
#pragma unroll
  for (int j = 0; j < kItems; ++j) {
    const uint32_t p = first + j * 256;
    if (p >= (uint32_t)a.pieces) break;
    const Cell e = cell(p, a.lc, a.inner);
    at[j] = e.c + e.inner * a.inner_stride + e.outer * a.outer_stride;
    x[j] = s[at[j]];
  }
#pragma unroll
  for (int j = 0; j < kItems; ++j) {
    if (first + j * 256 >= (uint32_t)a.pieces) break;
    d[at[j]] = x[j];
  }
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
  const int kv = (int)(b & 1);
  b >>= 1;
  const int g = (int)(b % a.G);
  const int r = (int)(b / a.G);
  const int len = a.lens[r], vis = a.vis_start[r];
  const int n = a.cu_vis[r + 1] - a.cu_vis[r], k = a.cu_keep[r + 1] - a.cu_keep[r];
  const int m = max(0, min(len - n + k, a.max_new));
  if (a.new_lens && tile == 0 && kv == 0 && g == 0 && threadIdx.x == 0) a.new_lens[r] = m;
  const int i0 = tile * kRowsPrune;
  if (i0 >= m) return;
  if (threadIdx.x < kRowsPrune) {
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
  uint4 *base = (uint4 *)(kv ? a.v : a.k) + g * a.layer_stride;
  // rows in the order they lie in: heads of a token, or tokens of a head
  const uint32_t inner = a.heads_inner ? a.Hkv : kRowsPrune;
  const uint32_t pieces = ((uint32_t)a.Hkv * kRowsPrune) << a.lc;
  for (uint32_t p0 = threadIdx.x; p0 < pieces; p0 += 256 * kItems) {
    uint4 x[kItems];
    int64_t at[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
      const uint32_t p = p0 + j * 256;
      at[j] = -1;
      if (p < pieces) {
        const Cell e = cell(p, a.lc, inner);
        const int head = a.heads_inner ? e.inner : e.outer, t = a.heads_inner ? e.outer : e.inner;
        const int64_t off = e.c + head * a.head_stride, s = from[t];
        if (to[t] >= 0) {
          at[j] = to[t] + off;
          x[j] = s >= 0 ? base[s + off] : make_uint4(0, 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kItems; ++j)
      if (at[j] >= 0) base[at[j]] = x[j];
  }
}

}  // namespace

namespace last {

int64_t copy_blocks(CopyArgs *a) {
  a->chunks = (a->pieces + 256 * kItems - 1) / (256 * kItems);
  return (int64_t)a->n * a->G * 2 * a->chunks;
}

hipError_t launch_cache_copy(const CopyArgs &a, int64_t blocks, hipStream_t s) {
  launch_begin("cache_copy", s);
  hipLaunchKernelGGL(k_cache_copy, dim3((unsigned)blocks), dim3(256), 0, s, a);
  return launch_end(s);
}

int64_t prune_blocks(PruneArgs *a) {
  a->tiles = std::max(1, (a->max_new + kRowsPrune - 1) / kRowsPrune);
  return (int64_t)a->R * a->G * 2 * a->tiles;
}

hipError_t launch_cache_prune(const PruneArgs &a, int64_t blocks, hipStream_t s) {
  launch_begin("cache_prune", s);
  hipLaunchKernelGGL(k_cache_prune, dim3((unsigned)blocks), dim3(256), 0, s, a);
  return launch_end(s);
}

}  // namespace last
