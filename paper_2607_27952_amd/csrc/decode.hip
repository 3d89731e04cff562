// Attention of one new token per sequence over a paged cache.
//
//   s_j = sigma q . k_j,  out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m)
//
// Bound: every cached key and value is read once for each 16 of the Hq / Hkv
// query heads that share it (17 to 32 read the cache twice), a few operations a
// byte, so the memory bounds it. All that matters is that enough 16-byte loads
// are in flight (a lane's share of a bf16 value row of 64 is 8 bytes); the
// matrix cores do the products because they make them nearly free.
// 64 sequences of 640 tokens with 32 + 32 heads of 128, 671 MB, take 104 us
// (6.4 TB/s; sums of rows by the framework that holds the tensors read 6.1).
//
// One wave takes 32 keys (bf16; 16 in fp32) at a time for up to 16 query heads
// that read one KV head, and everything stays in its registers:
//   S^T = K Q^T   A = K rows as they lie in memory, B = the heads (unused
//                 columns zero). The result has a head in each lane column,
//                 so a lane holds 8 (4) logits of one head.
//   O^T = V^T P^T B = P^T takes those logits' probabilities as they are: the
//                 order of the summed index is free as long as A agrees, so
//                 lane group j of V takes the keys 16 t + 4 j + r whose
//                 probabilities it already holds. A = V^T: lane m loads the
//                 elements d = w m + i (w = Dh / 16) of a key, whole rows
//                 across 16 lanes, and product i takes element i of each lane.
//                 In bf16 pairs of keys are packed by byte permutes.
// So neither P nor V passes through LDS. The softmax keeps a running maximum
// per head that moves only when a logit exceeds it (then all lanes of the
// head agree on the new one), and sums kept apart per lane until the end.
// In bf16 a probability enters whole, as the sum of three bf16 numbers of 8
// bits each, in three products. In two, the last 8 bits rounded off, 397
// outputs of 196608 were not the exact ones rounded (128 sequences of 288 to
// 16640 tokens), with three 57; the third product costs nothing beside the
// memory (the same batch 90.5 us with two, 90.4 with three; 64 sequences of 640
// tokens with 32 + 32 heads 103.9 and 104.0).
//
// The waves of a block take the tiles of its part of the sequence in turn and
// join through LDS; parts of a long sequence are joined by a second kernel, in
// the order of the parts.
#include <algorithm>

#include "last_internal.h"

namespace {

using last::DecodeArgs;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Keys and values are read once: past the caches.
template <typename V>
__device__ __forceinline__ V stream(const V *p) {
  return __builtin_nontemporal_load(p);
}

constexpr int kIds = last::kDecodeIds;
constexpr int W = 4;         // waves of a block
constexpr int kJoin = 256;   // threads of a joining block
constexpr float kLn2 = 0.6931471805599453f;

// A tile's operands and products for one element type.
template <typename T, int DH>
struct Tile;

template <int DH>
struct Tile<__bf16, DH> {
  static constexpr int kKeys = 32, kGroups = 2;   // keys of a tile, of 16 each
  static constexpr int kVec = DH / 16;            // elements of V a lane takes from a key
  static constexpr int kSteps = DH / 32;
  bf16x8 q[kSteps], k[kGroups][kSteps];
  uint32_t v[8][kVec / 2];
  __device__ __forceinline__ void load_q(const __bf16 *row, bool valid, int j) {
#pragma unroll
    for (int c = 0; c < kSteps; ++c)
      q[c] = valid ? *reinterpret_cast<const bf16x8 *>(row + 32 * c + 8 * j) : bf16x8{};
  }
  __device__ __forceinline__ void load_k(int t, const __bf16 *row, int j) {
#pragma unroll
    for (int c = 0; c < kSteps; ++c) k[t][c] = stream(reinterpret_cast<const bf16x8 *>(row + 32 * c + 8 * j));
  }
  __device__ __forceinline__ void load_v(int t, int r, const __bf16 *row, int m) {
    if constexpr (kVec == 8) {
      const u32x4 x = stream(reinterpret_cast<const u32x4 *>(row + 8 * m));
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * t + r][i] = x[i];
    } else {
      const u32x2 x = stream(reinterpret_cast<const u32x2 *>(row + 4 * m));
      v[4 * t + r][0] = x[0], v[4 * t + r][1] = x[1];
    }
  }
  __device__ __forceinline__ void zero_v(int t, int r) {
#pragma unroll
    for (int i = 0; i < kVec / 2; ++i) v[4 * t + r][i] = 0;
  }
  __device__ __forceinline__ f32x4 logits(int t) const {
    f32x4 s{};
#pragma unroll
    for (int c = 0; c < kSteps; ++c) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[t][c], q[c], s, 0, 0, 0);
    return s;
  }
  __device__ __forceinline__ void values(const float (&p)[8], f32x4 (&o)[kVec]) const {
    bf16x8 part[3];
    uint32_t b[8];
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = p[i];
#pragma unroll
    for (int c = 0; c < 3; ++c) {   // the leading 8 bits of what is left; no difference rounds
      uint4 w;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        b[i] = __float_as_uint(rest[i]);
        rest[i] -= __uint_as_float(b[i] & 0xFFFF0000u);
      }
      w.x = __builtin_amdgcn_perm(b[1], b[0], 0x07060302u);
      w.y = __builtin_amdgcn_perm(b[3], b[2], 0x07060302u);
      w.z = __builtin_amdgcn_perm(b[5], b[4], 0x07060302u);
      w.w = __builtin_amdgcn_perm(b[7], b[6], 0x07060302u);
      part[c] = __builtin_bit_cast(bf16x8, w);
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      uint4 w;   // element i of the 8 keys, two keys a word
      const uint32_t sel = (i & 1) ? 0x07060302u : 0x05040100u;
      w.x = __builtin_amdgcn_perm(v[1][i / 2], v[0][i / 2], sel);
      w.y = __builtin_amdgcn_perm(v[3][i / 2], v[2][i / 2], sel);
      w.z = __builtin_amdgcn_perm(v[5][i / 2], v[4][i / 2], sel);
      w.w = __builtin_amdgcn_perm(v[7][i / 2], v[6][i / 2], sel);
      const bf16x8 a = __builtin_bit_cast(bf16x8, w);
#pragma unroll
      for (int c = 0; c < 3; ++c) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, part[c], o[i], 0, 0, 0);
    }
  }
};

template <int DH>
struct Tile<float, DH> {
  static constexpr int kKeys = 16, kGroups = 1;
  static constexpr int kVec = DH / 16;
  static constexpr int kSteps = DH / 16;
  f32x4 q[kSteps], k[kSteps];
  float v[4][kVec];
  __device__ __forceinline__ void load_q(const float *row, bool valid, int j) {
#pragma unroll
    for (int c = 0; c < kSteps; ++c) q[c] = valid ? *reinterpret_cast<const f32x4 *>(row + 16 * c + 4 * j) : f32x4{};
  }
  __device__ __forceinline__ void load_k(int, const float *row, int j) {
#pragma unroll
    for (int c = 0; c < kSteps; ++c) k[c] = stream(reinterpret_cast<const f32x4 *>(row + 16 * c + 4 * j));
  }
  __device__ __forceinline__ void load_v(int, int r, const float *row, int m) {
#pragma unroll
    for (int c = 0; c < kVec; c += 4) {
      const f32x4 x = stream(reinterpret_cast<const f32x4 *>(row + kVec * m + c));
#pragma unroll
      for (int e = 0; e < 4; ++e) v[r][c + e] = x[e];
    }
  }
  __device__ __forceinline__ void zero_v(int, int r) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[r][i] = 0.f;
  }
  __device__ __forceinline__ f32x4 logits(int) const {
    f32x4 s{};
#pragma unroll
    for (int c = 0; c < kSteps; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c][e], q[c][e], s, 0, 0, 0);
    return s;
  }
  __device__ __forceinline__ void values(const float (&p)[4], f32x4 (&o)[kVec]) const {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][i], p[r], o[i], 0, 0, 0);
  }
};

__device__ __forceinline__ void store4(float *p, f32x4 v) { *reinterpret_cast<f32x4 *>(p) = v; }
__device__ __forceinline__ void store4(__bf16 *p, f32x4 v) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  bf16x4 b;
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = (__bf16)v[i];
  *reinterpret_cast<bf16x4 *>(p) = b;
}

__device__ __forceinline__ int clamp_len(const DecodeArgs &a, int r) { return max(0, min(a.lens[r], a.max_len)); }

// The waves of a block take tiles of keys of WH KV heads, W / WH tiles each: 1
// where a head's rows lie together, up to 4 where the heads of a token do.
//
// The work is one line of steps (a tile each wave): unit by unit (16 query
// heads on each of WH KV heads of a sequence), sequence by sequence. In a
// split call every block takes an equal stretch of the line (to one step),
// whatever the units it belongs to, by the lengths on the device: the blocks
// have the same work however ragged the batch, and none is without.
struct Share {
  int each, more;   // steps of a block; blocks from the first on that have one more
  __device__ __forceinline__ Share(int total, int blocks) : each(total / blocks), more(total - each * blocks) {}
  __device__ __forceinline__ int start(int b) const { return b * each + min(b, more); }
  __device__ __forceinline__ int block_of(int step) const {
    const int head = more * (each + 1);
    return step < head ? step / (each + 1) : more + (step - head) / each;
  }
};
// Inclusive sums over a wave, whose sum is returned in `sum`: DPP shifts inside
// rows of 16 lanes, then the rows' ends. It stands before a block's first load:
// one sequence of 2048 tokens 9.6 us, 10.0 with shuffles, which pass LDS.
__device__ __forceinline__ int wave_scan(int v, int *sum) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
  const int a = __builtin_amdgcn_readlane(v, 15), b = a + __builtin_amdgcn_readlane(v, 31);
  const int c = b + __builtin_amdgcn_readlane(v, 47), row = (threadIdx.x & 63) >> 4;
  *sum = c + __builtin_amdgcn_readlane(v, 63);
  return v + (row == 0 ? 0 : row == 1 ? a : row == 2 ? b : c);
}

// Where a block's stretch begins: its sequence, the line's steps before that
// sequence, and the line's length. Called by whole waves.
struct Start {
  int r, before, total;
};
template <int STEP>
__device__ __forceinline__ Start find_start(const DecodeArgs &a, int units, int block) {
  const int lane = threadIdx.x & 63;
  auto steps = [&](int r) { return r < a.R ? units * ((clamp_len(a, r) + STEP - 1) / STEP) : 0; };
  int n = steps(lane), sum, total;   // of the first 64 sequences, which are often all
  int x = wave_scan(n, &sum);
  total = sum;
  if (a.R > 64) {
    int rest = 0, more;
    for (int r = 64 + lane; r < a.R; r += 64) rest += steps(r);
    wave_scan(rest, &more);
    total += more;
  }
  const int at = Share(total, a.blocks).start(block);
  int base = 0;
  for (int r0 = 0; r0 < a.R; r0 += 64) {
    if (r0) x = wave_scan(n = steps(r0 + lane), &sum);
    const unsigned long long behind = __ballot(base + x > at);
    if (behind) {
      const int l = __ffsll((long long)behind) - 1;
      return Start{r0 + l, base + __builtin_amdgcn_readlane(x - n, l), total};
    }
    base += sum;
  }
  return Start{a.R, base, total};   // behind the line's end
}

template <typename T, int DH, int WH>
__global__ __launch_bounds__(64 * W) void k_decode(DecodeArgs a) {
  using TL = Tile<T, DH>;
  constexpr int KEYS = TL::kKeys, GR = TL::kGroups, VEC = TL::kVec, NP = 4 * GR, WK = W / WH, STEP = WK * KEYS;
  constexpr int ROW = DH + 4;   // padded, or the 16 heads of a wave's result share a bank
  __shared__ int32_t ids[kIds];
  __shared__ float so[W][16 * ROW];
  __shared__ float sm[W][16], sl[W][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, j = lane >> 4;
  const int units = a.head_tiles * (a.Hkv / WH), lg = a.lg_page;

  int r, unit, t0 = 0, left, total = 0;   // the segment's sequence, unit and first step; steps of this block
  if (a.split) {
    const Start s = find_start<STEP>(a, units, blockIdx.x);
    const Share share(total = s.total, a.blocks);
    const int at = share.start(blockIdx.x);
    left = share.start(blockIdx.x + 1) - at;
    if (left <= 0) return;
    r = s.r;
    const int n = (clamp_len(a, r) + STEP - 1) / STEP;
    unit = (at - s.before) / n;
    t0 = at - s.before - unit * n;
  } else {
    r = blockIdx.x / units;
    unit = blockIdx.x - r * units;
    left = max(1, (clamp_len(a, r) + STEP - 1) / STEP);
  }

  for (bool first = true;; first = false) {
    const int kv0 = unit / a.head_tiles * WH, ht = unit - kv0 / WH * a.head_tiles;
    const int heads = min(16, a.group - 16 * ht);   // of this unit, on each of its WH KV heads
    const int kvh = kv0 + wave / WK, h0 = kvh * a.group + 16 * ht;
    const int len = clamp_len(a, r);
    const int steps = (len + STEP - 1) / STEP, t1 = min(steps, t0 + left);
    // query head h of KV head kv0 + w, as a row of out and lse
    auto head_row = [&](int w, int h) -> int64_t { return (int64_t)r * a.Hq + (kv0 + w) * a.group + 16 * ht + h; };
    if (!a.split && len == 0) {   // nothing to attend to
      for (int x = threadIdx.x; x < WH * heads * (DH / 4); x += 64 * W) {
        const int y = x / (DH / 4), w = y / heads;
        const int64_t at = head_row(w, y - w * heads);
        store4((T *)a.out + at * DH + 4 * (x % (DH / 4)), f32x4{});
        if (a.lse && x % (DH / 4) == 0) a.lse[at] = -INFINITY;
      }
      return;
    }
    const T *kb = (const T *)a.k + kvh * a.head_stride, *vb = (const T *)a.v + kvh * a.head_stride;
    TL t;
    t.load_q((const T *)a.q + r * a.q_stride + (int64_t)(h0 + min(col, heads - 1)) * DH, col < heads, j);
    float m = -INFINITY, l = 0.f;
    f32x4 o[VEC] = {};
    int bad = 0;
    const int end = min(len, t1 * STEP);
    for (int n0 = t0 * STEP, n1; n0 < end; n0 = n1) {
      // the ids of as many pages as there is room for; one outside the cache
      // is not followed and spoils the result
      n1 = (int)min<int64_t>(end, n0 + ((int64_t)(kIds - 1) << lg) / STEP * STEP);
      const int page0 = n0 >> lg, pages = ((n1 - 1) >> lg) - page0 + 1;
      if (n0 > t0 * STEP) __syncthreads();
      for (int i = threadIdx.x; i < pages; i += 64 * W) {
        int32_t id = a.table[(int64_t)r * a.max_pages + page0 + i];
        if ((uint32_t)id >= (uint32_t)a.n_pages) id = 0, bad = 1;
        ids[i] = id;
      }
      __syncthreads();
      auto row = [&](int key) -> int64_t {
        key = min(key, n1 - 1);
        return ids[(key >> lg) - page0] * a.page_stride + (key & ((1 << lg) - 1)) * a.token_stride;
      };
      const int k0w = n0 + wave % WK * KEYS;
      if (k0w < n1) {
#pragma unroll
        for (int g = 0; g < GR; ++g) t.load_k(g, kb + row(k0w + 16 * g + col), j);
      }
      for (int k0 = k0w; k0 < n1; k0 += STEP) {
#pragma unroll
        for (int g = 0; g < GR; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) t.load_v(g, i, vb + row(k0 + 16 * g + 4 * j + i), col);
        float p[NP];
        float top = -INFINITY;
#pragma unroll
        for (int g = 0; g < GR; ++g) {
          const f32x4 s = t.logits(g);
#pragma unroll
          for (int i = 0; i < 4; ++i) p[4 * g + i] = s[i] * a.scale_log2;
        }
        if (k0 + STEP < n1) {   // the next tile's keys, into the registers just read
#pragma unroll
          for (int g = 0; g < GR; ++g) t.load_k(g, kb + row(k0 + STEP + 16 * g + col), j);
        }
        if (k0 + KEYS > n1) {   // keys behind the end: no weight, and nothing of what lies there
#pragma unroll
          for (int g = 0; g < GR; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (k0 + 16 * g + 4 * j + i >= n1) {
                p[4 * g + i] = -INFINITY;
                t.zero_v(g, i);
              }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) top = fmaxf(top, p[i]);
        if (__any(top > m)) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float next = fmaxf(m, top);
          const float f = m == next ? 1.f : __builtin_amdgcn_exp2f(m - next);
          m = next;
          l *= f;
#pragma unroll
          for (int i = 0; i < VEC; ++i) o[i] *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m;   // every logit so far -inf: weights 0
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          p[i] = __builtin_amdgcn_exp2f(p[i] - ref);
          l += p[i];
        }
        t.values(p, o);
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // join the waves: O^T row 4 j + r of product i is element d = VEC (4 j + r) + i
    if (j == 0) sm[wave][col] = m, sl[wave][col] = l;
    if (col < heads) {
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
#pragma unroll
        for (int i = 0; i < VEC; i += 4)
          *reinterpret_cast<f32x4 *>(&so[wave][col * ROW + VEC * (4 * j + r4) + i]) =
              f32x4{o[i][r4], o[i + 1][r4], o[i + 2][r4], o[i + 3][r4]};
    }
    bad = __syncthreads_or(bad);
    const bool whole = t0 == 0 && t1 == steps;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (first ? 0 : 1);   // a block has two parts at most
    for (int x = threadIdx.x; x < WH * heads * (DH / 4); x += 64 * W) {
      const int y = x / (DH / 4), hw = y / heads, h = y - hw * heads, d = 4 * (x % (DH / 4));
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < WK; ++w) top = fmaxf(top, sm[hw * WK + w][h]);
      const float ref = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
      f32x4 acc{};
#pragma unroll
      for (int w = 0; w < WK; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm[hw * WK + w][h] - ref);
        sum += f * sl[hw * WK + w][h];
        acc += f * *reinterpret_cast<const f32x4 *>(&so[hw * WK + w][h * ROW + d]);
      }
      if (bad) sum = NAN;
      if (whole) {
        const int64_t at = head_row(hw, h);
        store4((T *)a.out + at * DH + d, acc / sum);
        if (a.lse && d == 0) a.lse[at] = (ref + __builtin_amdgcn_logf(sum)) * kLn2;
      } else {
        const int64_t at = (slot * WH + hw) * 16 + h;
        *reinterpret_cast<f32x4 *>(a.part_o + at * DH + d) = acc;
        if (d == 0) a.part_ml[at] = make_float2(top, sum);
      }
    }
    if (a.split && t0 == 0 && threadIdx.x == 0) {   // where the unit's parts are: the join's
      int parts = 1;
      if (!whole) {
        const Share share(total, a.blocks);
        parts = share.block_of(share.start(blockIdx.x + 1) - left + steps - 1) - (int)blockIdx.x + 1;
      }
      a.info[(int64_t)r * units + unit] = make_int2((int)slot, parts);
    }
    left -= t1 - t0;
    if (left <= 0) return;
    t0 = 0;
    if (++unit == units) {
      unit = 0;
      do ++r;
      while (r < a.R && clamp_len(a, r) == 0);
      if (r >= a.R) return;
    }
  }
}

// The parts of one query head joined, in the order of the blocks that left
// them (a block's first part is in slot 2 b, its last one, unless that is its
// first, in 2 b + 1): a set of DH / 4 lanes takes every SETS-th part, then the
// sets are added in order. Sequences of length 0 get their zeros here.
template <typename T, int DH>
__global__ __launch_bounds__(kJoin) void k_decode_join(DecodeArgs a) {
  constexpr int LANES = DH / 4, SETS = kJoin / LANES, AHEAD = 4;
  __shared__ f32x4 so[SETS][LANES];
  __shared__ float sm[SETS], sl[SETS];
  const int64_t hq = blockIdx.x;
  const int r = (int)(hq / a.Hq), h = (int)(hq - (int64_t)r * a.Hq);
  const int e = threadIdx.x % LANES, set = threadIdx.x / LANES;
  const int kvh = h / a.group, ht = (h - kvh * a.group) / 16, col = (h - kvh * a.group) % 16;
  const int WH = a.heads_of_block;
  const int2 info = a.info[(int64_t)r * (a.head_tiles * (a.Hkv / WH)) + kvh / WH * a.head_tiles + ht];
  if (clamp_len(a, r) == 0) {   // info is not set
    if (set == 0) store4((T *)a.out + hq * DH + 4 * e, f32x4{});
    if (a.lse && threadIdx.x == 0) a.lse[hq] = -INFINITY;
    return;
  }
  const int parts = info.y;
  if (parts == 1) return;   // written by its block
  float m = -INFINITY, l = 0.f;
  f32x4 acc{};
  for (int i0 = set; i0 < parts; i0 += AHEAD * SETS) {
    float2 x[AHEAD];
    f32x4 o[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {   // all loads before the first use; behind the end the last part again
      const int i = min(i0 + u * SETS, parts - 1);
      const int64_t at = ((i == 0 ? (int64_t)info.x : 2 * ((int64_t)(info.x >> 1) + i)) * WH + kvh % WH) * 16 + col;
      x[u] = a.part_ml[at];
      o[u] = *reinterpret_cast<const f32x4 *>(a.part_o + at * DH + 4 * e);
      if (i0 + u * SETS >= parts) x[u] = make_float2(-INFINITY, 0.f), o[u] = f32x4{};
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) top = fmaxf(top, x[u].x);
    const float ref = top == -INFINITY ? 0.f : top, f = __builtin_amdgcn_exp2f(m - ref);
    l *= f;
    acc *= f;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const float g = __builtin_amdgcn_exp2f(x[u].x - ref);
      l += x[u].y * g;
      acc += o[u] * g;
    }
    m = top;
  }
  so[set][e] = acc;
  if (e == 0) sm[set] = m, sl[set] = l;
  __syncthreads();
  if (set == 0) {
    float top = m;
#pragma unroll
    for (int i = 1; i < SETS; ++i) top = fmaxf(top, sm[i]);
    const float ref = top == -INFINITY ? 0.f : top;
    acc = f32x4{}, l = 0.f;
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
      const float f = __builtin_amdgcn_exp2f(sm[i] - ref);
      acc += f * so[i][e];
      l += f * sl[i];
    }
    store4((T *)a.out + hq * DH + 4 * e, acc / l);
    if (a.lse && e == 0) a.lse[hq] = (ref + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

template <typename T, int DH>
hipError_t launch_t(const DecodeArgs &a, hipStream_t s) {
  last::launch_begin("decode", s);
  const dim3 grid((unsigned)a.blocks), block(64 * W);
  if (a.heads_of_block == 2) hipLaunchKernelGGL((k_decode<T, DH, 2>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_decode<T, DH, 1>), grid, block, 0, s, a);
  hipError_t e = last::launch_end(s);
  if (e != hipSuccess || !a.split) return e;
  last::launch_begin("decode_join", s);
  hipLaunchKernelGGL((k_decode_join<T, DH>), dim3((unsigned)(a.R * a.Hq)), dim3(kJoin), 0, s, a);
  return last::launch_end(s);
}

}  // namespace

namespace last {

// How a call is laid out: by the bounds of the lengths alone, so that a
// captured call may be replayed with any lengths within them.
//
// Split or not, in steps: one block a unit ends not before the longest unit,
// and after about `fair` steps (what a compute unit gets if all get the same)
// and half the longest's excess over the mean. Splitting takes `fair` and the
// join, which costs about what 3 steps of an idle chip do; the tenth is for
// its blocks' search of their start. More waves a block do not shorten a unit:
// one compute unit reads some 40 GB/s, whatever it has in flight. Both, split
// first, us:
//   64 sequences of 640, 32 + 32 heads       110   104
//    8 of 4096, 32 + 32 heads                 86    81
//    4 of 1000, 32 + 32 heads               18.6  20.6
//  200 of 8 to 700, 32 on 8 heads             43    40
//   32 of 500, 32 on 8 heads                19.3  15.0
//    1 of 104, fp32, 16 + 16 heads of 64     9.4   6.9
//    4 of 300, 28 on 4 heads                 9.7   9.0
//    1 of 640, 28 on 4 heads                 9.7  13.5
//   16 of 1000, 28 on 4 heads               14.8  20.2
//    8 of 16512, 28 on 4 heads                54   455
//  128 of 288 to 16640, 12 on 2 heads         89   229
// The bounds may be far above the lengths, which an unsplit call would meet
// with one long block: it is not used past 16 steps. 64 sequences with bounds
// of 8192, 28 on 4 heads, one of them that long and 500 tokens in the others:
// split 23 us, not split 116 (what this costs is the 5 of the second line);
// 256 slots with bounds of 0 but for one of 20000, 12 on 2 heads: 16 and 261.
//
// A split call has two blocks a compute unit, what its 212 to 220 registers let
// live there with heads of 128: with one the ragged 200 take 57 us for 44, with
// four the 8 of 16512 take 58 for 54. Heads of 64 take 136 to 152, of which three
// blocks would fit; they have two all the same.
//
// Keys of two KV heads beside each other in memory go to one block: 8 of 16512
// 54 us against 57, 64 of 640 107 against 118 where the heads of a token lie
// together; four at a time was no better.
DecodePlan make_decode_plan(const last_cache *c, const last_pages *p, int32_t Hq) {
  DecodePlan d{};
  const bool beside = c->Hkv > 1 && c->head_stride < c->token_stride;
  d.heads_of_block = beside && c->Hkv % 2 == 0 ? 2 : 1;
  const int64_t step = W / d.heads_of_block * (c->dtype == LAST_BF16 ? 32 : 16);   // keys
  int64_t total = 0;
  for (int32_t r = 0; r < p->R; ++r) {
    total += (p->lens_h[r] + step - 1) / step;
    d.max_len = std::max(d.max_len, p->lens_h[r]);
  }
  d.head_tiles = (Hq / c->Hkv + 15) / 16;
  const int64_t per_seq = (int64_t)(c->Hkv / d.heads_of_block) * d.head_tiles, units = p->R * per_seq;
  total *= per_seq;
  const int64_t longest = (d.max_len + step - 1) / step;
  const int64_t room = 2 * device_cus();   // blocks the chip holds at once
  const int64_t fair = 10 * total / device_cus(), tail = 10 * longest - 10 * total / units;   // in tenths
  d.split = longest > 16 || (total > units && std::max(10 * longest, fair + tail / 2) > fair + fair / 10 + 30);
  d.shares = std::max<int64_t>(1, std::min(total, room));
  d.blocks = d.split ? d.shares : units;
  d.steps = units * longest;
  return d;
}

hipError_t launch_decode(const DecodeArgs &a, last_dtype dtype, int32_t Dh, hipStream_t s) {
  if (dtype == LAST_F32) return Dh == 64 ? launch_t<float, 64>(a, s) : launch_t<float, 128>(a, s);
  return Dh == 64 ? launch_t<__bf16, 64>(a, s) : launch_t<__bf16, 128>(a, s);
}

}  // namespace last
