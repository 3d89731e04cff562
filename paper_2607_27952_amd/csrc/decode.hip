// Attention of one new token per sequence over a paged cache.
//
//   s_j = sigma q . k_j,  out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m)
//
// Bound: every cached key and value is read once and used for the Hq / Hkv
// query heads that share it, a few operations a byte, so the memory bounds it.
// All that matters is that enough 16-byte loads are in flight; the matrix
// cores do the products because they make them nearly free.
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
// In bf16 a probability enters as hi + lo, two bf16 numbers, in two products:
// the output's error is then that of its own rounding.
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

constexpr int kWaves = 4;
constexpr int kIds = last::kDecodeIds;
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
    for (int c = 0; c < kSteps; ++c) k[t][c] = *reinterpret_cast<const bf16x8 *>(row + 32 * c + 8 * j);
  }
  __device__ __forceinline__ void load_v(int t, int r, const __bf16 *row, int m) {
    if constexpr (kVec == 8) {
      const uint4 x = *reinterpret_cast<const uint4 *>(row + 8 * m);
      v[4 * t + r][0] = x.x, v[4 * t + r][1] = x.y, v[4 * t + r][2] = x.z, v[4 * t + r][3] = x.w;
    } else {
      const uint2 x = *reinterpret_cast<const uint2 *>(row + 4 * m);
      v[4 * t + r][0] = x.x, v[4 * t + r][1] = x.y;
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
    bf16x8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      hi[i] = (__bf16)p[i];
      lo[i] = (__bf16)(p[i] - (float)hi[i]);
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
      o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, hi, o[i], 0, 0, 0);
      o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, lo, o[i], 0, 0, 0);
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
    for (int c = 0; c < kSteps; ++c) k[c] = *reinterpret_cast<const f32x4 *>(row + 16 * c + 4 * j);
  }
  __device__ __forceinline__ void load_v(int, int r, const float *row, int m) {
#pragma unroll
    for (int c = 0; c < kVec; c += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4 *>(row + kVec * m + c);
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

template <typename T, int DH>
__global__ __launch_bounds__(64 * kWaves) void k_decode(DecodeArgs a) {
  using TL = Tile<T, DH>;
  constexpr int KEYS = TL::kKeys, GR = TL::kGroups, VEC = TL::kVec, NP = 4 * GR;
  constexpr int ROW = DH + 4;   // padded, or the 16 heads of a wave's result share a bank
  __shared__ int32_t ids[kIds];
  __shared__ float so[kWaves][16 * ROW];
  __shared__ float sm[kWaves][16], sl[kWaves][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, j = lane >> 4;
  const int part = blockIdx.x % a.parts;
  const int unit = blockIdx.x / a.parts;
  const int ht = unit % a.head_tiles, kvh = (unit / a.head_tiles) % a.Hkv, r = unit / (a.head_tiles * a.Hkv);
  const int heads = min(16, a.group - 16 * ht);   // of this block
  const int h0 = kvh * a.group + 16 * ht;
  const int len = max(0, min(a.lens[r], a.max_len));
  const int n0 = part * a.keys, n1 = min(len, n0 + a.keys);
  T *out = (T *)a.out + ((int64_t)r * a.Hq + h0) * DH;
  if (n0 >= n1) {
    if (len == 0 && part == 0) {   // nothing to attend to
      for (int i = threadIdx.x; i < heads * (DH / 4); i += 64 * kWaves) store4(out + 4 * i, f32x4{});
      if (a.lse && (int)threadIdx.x < heads) a.lse[(int64_t)r * a.Hq + h0 + threadIdx.x] = -INFINITY;
    }
    return;
  }

  // the part's pages; one outside the cache is not followed and spoils the result
  const int lg = a.lg_page, first = n0 >> lg, pages = ((n1 - 1) >> lg) - first + 1;
  int bad = 0;
  for (int i = threadIdx.x; i < pages; i += 64 * kWaves) {
    int32_t id = a.table[(int64_t)r * a.max_pages + first + i];
    if ((uint32_t)id >= (uint32_t)a.n_pages) id = 0, bad = 1;
    ids[i] = id;
  }
  bad = __syncthreads_or(bad);

  const T *kb = (const T *)a.k + kvh * a.head_stride, *vb = (const T *)a.v + kvh * a.head_stride;
  auto row = [&](int key) -> int64_t {
    key = min(key, n1 - 1);
    return ids[(key >> lg) - first] * a.page_stride + (key & ((1 << lg) - 1)) * a.token_stride;
  };
  TL t;
  t.load_q((const T *)a.q + r * a.q_stride + (int64_t)(h0 + min(col, heads - 1)) * DH, col < heads, j);
  float m = -INFINITY, l = 0.f;
  f32x4 o[VEC] = {};
  for (int k0 = n0 + wave * KEYS; k0 < n1; k0 += kWaves * KEYS) {
#pragma unroll
    for (int g = 0; g < GR; ++g) t.load_k(g, kb + row(k0 + 16 * g + col), j);
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
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (bad) l = NAN;

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
  __syncthreads();
  for (int x = threadIdx.x; x < heads * (DH / 4); x += 64 * kWaves) {
    const int h = x / (DH / 4), d = 4 * (x % (DH / 4));
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm[w][h]);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    f32x4 acc{};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm[w][h] - ref);
      sum += f * sl[w][h];
      acc += f * *reinterpret_cast<const f32x4 *>(&so[w][h * ROW + d]);
    }
    const int64_t hq = (int64_t)r * a.Hq + h0 + h;
    if (a.parts == 1) {
      store4(out + h * DH + d, acc / sum);
      if (a.lse && d == 0) a.lse[hq] = (ref + __builtin_amdgcn_logf(sum)) * kLn2;
    } else {
      *reinterpret_cast<f32x4 *>(a.part_o + (hq * a.parts + part) * DH + d) = acc;
      if (d == 0) a.part_ml[hq * a.parts + part] = make_float2(top, sum);
    }
  }
}

// The parts of one query head joined: a wave takes every 4th part for its
// lanes' elements, in order, and the waves are added in order.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_decode_join(DecodeArgs a) {
  constexpr int LANES = DH / 4, SETS = 256 / LANES;
  __shared__ f32x4 so[SETS][LANES];
  __shared__ float st[4], ss[SETS];
  const int64_t hq = blockIdx.x;
  const int r = (int)(hq / a.Hq);
  const int len = max(0, min(a.lens[r], a.max_len));
  const int n = (len + a.keys - 1) / a.keys;
  if (n == 0) return;   // written by the part kernel
  const float2 *ml = a.part_ml + hq * a.parts;
  float top = -INFINITY;
  for (int i = threadIdx.x; i < n; i += 256) top = fmaxf(top, ml[i].x);
  top = last_dev::wave_max(top);
  if ((threadIdx.x & 63) == 0) st[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(st[0], st[1]), fmaxf(st[2], st[3]));
  const float ref = top == -INFINITY ? 0.f : top;
  const int e = threadIdx.x % LANES, set = threadIdx.x / LANES;
  f32x4 acc{};
  float sum = 0.f;
#pragma unroll 4
  for (int i = set; i < n; i += SETS) {
    const float2 x = ml[i];
    const float f = __builtin_amdgcn_exp2f(x.x - ref);
    sum += f * x.y;
    acc += f * *reinterpret_cast<const f32x4 *>(a.part_o + (hq * a.parts + i) * DH + 4 * e);
  }
  so[set][e] = acc;
  if (e == 0) ss[set] = sum;
  __syncthreads();
  if (set == 0) {
#pragma unroll
    for (int i = 1; i < SETS; ++i) {
      acc += so[i][e];
      sum += ss[i];
    }
    store4((T *)a.out + hq * DH + 4 * e, acc / sum);
    if (a.lse && e == 0) a.lse[hq] = (ref + __builtin_amdgcn_logf(sum)) * kLn2;
  }
}

template <typename T, int DH>
hipError_t launch_t(const DecodeArgs &a, hipStream_t s) {
  last::launch_begin("decode", s);
  const unsigned blocks = (unsigned)(a.R * a.Hkv * a.head_tiles * a.parts);
  hipLaunchKernelGGL((k_decode<T, DH>), dim3(blocks), dim3(64 * kWaves), 0, s, a);
  hipError_t e = last::launch_end(s);
  if (e != hipSuccess || a.parts == 1) return e;
  last::launch_begin("decode_join", s);
  hipLaunchKernelGGL((k_decode_join<T, DH>), dim3((unsigned)(a.R * a.Hq)), dim3(256), 0, s, a);
  return last::launch_end(s);
}

}  // namespace

namespace last {

// How a call is split: by the bounds of the lengths alone, so that a captured
// call may be replayed with any lengths within them.
DecodePlan make_decode_plan(const last_cache *c, const last_pages *p, int32_t Hq) {
  DecodePlan d{};
  int64_t total = 0;
  for (int32_t r = 0; r < p->R; ++r) {
    total += p->lens_h[r];
    d.max_len = std::max(d.max_len, p->lens_h[r]);
  }
  d.head_tiles = (Hq / c->Hkv + 15) / 16;
  const int64_t tile = kWaves * (c->dtype == LAST_BF16 ? 32 : 16);
  const int64_t work = total * c->Hkv * d.head_tiles;
  int64_t keys = work / (8 * device_cus());
  keys = std::max<int64_t>((keys + tile - 1) / tile * tile, 2 * tile);
  keys = std::min<int64_t>(keys, (int64_t)(kDecodeIds - 1) * c->page_size);
  keys = keys / tile * tile;
  if (d.max_len <= 512 && d.max_len <= keys * 4 && (int64_t)d.max_len <= (int64_t)(kDecodeIds - 1) * c->page_size)
    keys = std::max<int64_t>(keys, (d.max_len + tile - 1) / tile * tile);
  d.keys = (int32_t)keys;
  d.parts = (int32_t)std::max<int64_t>(1, (d.max_len + keys - 1) / keys);
  d.blocks = (int64_t)p->R * c->Hkv * d.head_tiles * d.parts;
  return d;
}

hipError_t launch_decode(const DecodeArgs &a, last_dtype dtype, int32_t Dh, hipStream_t s) {
  if (dtype == LAST_F32) return Dh == 64 ? launch_t<float, 64>(a, s) : launch_t<float, 128>(a, s);
  return Dh == 64 ? launch_t<__bf16, 64>(a, s) : launch_t<__bf16, 128>(a, s);
}

}  // namespace last
