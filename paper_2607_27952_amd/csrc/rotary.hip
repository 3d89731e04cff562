// Rotary positions with several axes (time, height, width), on rows of heads
// and, for a cache, with the turned keys and the values put into its pages.
//
//   a_i = pos[axis_i] inv_freq_i;  (x, y) -> (x cos a - y sin a, y cos a + x sin a)
//
// Angles: a position is an integer of up to 31 bits and a frequency an fp32
// number, so the angle is formed in 64 bits, in turns (a / 2 pi), reduced to
// the nearest whole turn there (2^31 turns leave 2^-22 of a turn), and only the
// remainder is rounded to fp32. Each angle is computed once per token, layer
// and block and serves every head: one sine and cosine for up to 64 pairs.
//
// The work is a copy, bound by the memory: each row is read once and written
// once, 32 bytes a thread, as the two 16-byte pieces whose elements pair up.
// 5.7 to 6.1 TB/s on 0.5 GB and more, where a copy of 1 GiB by the framework
// that holds the tensors reaches 5.2.
#include <algorithm>

#include "last_internal.h"

namespace {

using last::RotaryArgs;

constexpr int kTokens = 4;   // most tokens of a block

template <typename T>
struct Piece;   // 16 bytes as floats
template <>
struct Piece<float> {
  static constexpr int kN = 4;
  typedef float vec __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ void get(const vec v, float (&x)[kN]) {
#pragma unroll
    for (int i = 0; i < kN; ++i) x[i] = v[i];
  }
  static __device__ __forceinline__ vec put(const float (&x)[kN]) {
    vec v;
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = x[i];
    return v;
  }
};
template <>
struct Piece<__bf16> {
  static constexpr int kN = 8;
  typedef __bf16 vec __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ void get(const vec v, float (&x)[kN]) {
#pragma unroll
    for (int i = 0; i < kN; ++i) x[i] = (float)v[i];
  }
  static __device__ __forceinline__ vec put(const float (&x)[kN]) {
    vec v;
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = (__bf16)x[i];   // to nearest even, once
    return v;
  }
};

// Where token t of the new ones is stored, in elements from its layer's start;
// -1 where it is not. Called by whole waves: its sequence is found with 64
// probes a level.
__device__ int64_t cache_place(const RotaryArgs &a, int t) {
  int r = t, first = t, count = 1;
  if (a.cu_new) {
    int lo = 0, hi = a.R;   // the largest r with cu_new[r] <= t is in [lo, hi)
    while (hi - lo > 1) {
      const int step = (hi - lo + 63) / 64, at = lo + (int)(threadIdx.x & 63) * step;
      const unsigned long long ok = __ballot(at < hi && a.cu_new[at] <= t);
      if (!ok) return -1;
      lo += (63 - __clzll((long long)ok)) * step;
      hi = min(hi, lo + step);
    }
    r = lo;
    first = a.cu_new[r];
    count = a.cu_new[r + 1] - first;
    if (t < first || t - first >= count) return -1;
  }
  const int64_t at = (int64_t)a.lens[r] - count + (t - first);
  if (at < 0 || at >= a.max_len) return -1;
  const int32_t page = a.table[(int64_t)r * a.max_pages + (at >> a.lg_page)];
  if ((uint32_t)page >= (uint32_t)a.n_pages) return -1;
  return page * a.page_stride + (at & ((1 << a.lg_page) - 1)) * a.slot_stride;
}

template <typename T, int DH, bool APPEND>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a) {
  constexpr int VEC = Piece<T>::kN;
  constexpr int NC = DH / VEC / 2;       // 32-byte items of a row
  constexpr int ROWS = 256 / NC;         // rows of a step
  __shared__ float cs[kTokens][64], sn[kTokens][64];
  __shared__ int64_t place[kTokens];
  const int part = blockIdx.x % a.parts;
  const int64_t rest = blockIdx.x / a.parts;
  const int g = (int)(rest % a.G);
  const int t0 = (int)(rest / a.G) * a.tokens;
  const int nt = min(a.tokens, a.T - t0);
  for (int i = threadIdx.x; i < nt * a.F; i += 256) {
    const int t = i / a.F, f = i - t * a.F;
    const double turns = (double)a.pos[(int64_t)a.axis[f] * a.T + t0 + t] * ((double)a.inv_freq[f] * 0.15915494309189535);
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    cs[t][f] = c;
    sn[t][f] = a.inverse ? -s : s;
  }
  if (APPEND)
    for (int t = threadIdx.x / 64; t < nt; t += 4) {
      const int64_t at = cache_place(a, t0 + t);
      if (threadIdx.x % 64 == 0) place[t] = at;
    }
  __syncthreads();

  const int heads = a.Hq + (APPEND ? 2 : 1) * a.Hkv;
  const int h0 = (int)((int64_t)heads * part / a.parts), span = (int)((int64_t)heads * (part + 1) / a.parts) - h0;
  const int ic = threadIdx.x % NC;
  int t = 0, h = threadIdx.x / NC;
  for (;; h += ROWS) {
    while (h >= span && t < nt) h -= span, ++t;
    if (t >= nt) break;
    const int head = h0 + h;
    const T *src;
    T *dst;
    bool turn = true;
    if (head < a.Hq) {
      src = (const T *)a.q + g * a.q_ls + (int64_t)(t0 + t) * a.q_ts + head * DH;
      dst = (T *)a.q_out + g * a.qo_ls + (int64_t)(t0 + t) * a.qo_ts + head * DH;
    } else {
      const int kh = head - a.Hq;
      if (APPEND) {
        const int64_t at = place[t];
        if (at < 0) continue;
        turn = kh < a.Hkv;
        const int hh = turn ? kh : kh - a.Hkv;
        const T *base = turn ? (const T *)a.k + g * a.k_ls + (int64_t)(t0 + t) * a.k_ts
                             : (const T *)a.v + g * a.v_ls + (int64_t)(t0 + t) * a.v_ts;
        src = base + hh * DH;
        dst = (T *)(turn ? a.k_out : a.v_out) + g * a.ko_ls + at + hh * a.head_stride;
      } else {
        src = (const T *)a.k + g * a.k_ls + (int64_t)(t0 + t) * a.k_ts + kh * DH;
        dst = (T *)a.k_out + g * a.ko_ls + (int64_t)(t0 + t) * a.ko_ts + kh * DH;
      }
    }
    // the item's two pieces: a pair of halves, or neighbours
    const int half = a.F / VEC;
    const bool halves = !a.adjacent && ic < half;
    const int p0 = halves ? ic : 2 * ic;
    const int p1 = halves ? ic + half : p0 + 1;
    typedef typename Piece<T>::vec vec;
    vec u0 = *reinterpret_cast<const vec *>(src + p0 * VEC), u1 = *reinterpret_cast<const vec *>(src + p1 * VEC);
    // What is not turned is stored as it was read: through fp32 and back a bf16
    // signalling NaN would change.
    if (turn && (halves || (a.adjacent && p0 * VEC < 2 * a.F))) {
      float x[VEC], y[VEC];
      Piece<T>::get(u0, x);
      Piece<T>::get(u1, y);
      if (halves) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float c = cs[t][p0 * VEC + e], s = sn[t][p0 * VEC + e];
          const float u = x[e] * c - y[e] * s;
          y[e] = y[e] * c + x[e] * s;
          x[e] = u;
        }
      } else {
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          const int f = (p0 * VEC + e) / 2, f1 = f + VEC / 2;
          const float u = x[e] * cs[t][f] - x[e + 1] * sn[t][f];
          x[e + 1] = x[e + 1] * cs[t][f] + x[e] * sn[t][f];
          x[e] = u;
          const float w = y[e] * cs[t][f1] - y[e + 1] * sn[t][f1];
          y[e + 1] = y[e + 1] * cs[t][f1] + y[e] * sn[t][f1];
          y[e] = w;
        }
      }
      u0 = Piece<T>::put(x);
      u1 = Piece<T>::put(y);
    }
    // Past the caches where the rows go to pages (appending 108000 tokens of
    // 12 + 2 heads 154 against 160 us), not where they stay rows (132096 tokens
    // of 28 + 4 heads 354 against 363).
    vec *d0 = reinterpret_cast<vec *>(dst + p0 * VEC), *d1 = reinterpret_cast<vec *>(dst + p1 * VEC);
    if (APPEND) {
      __builtin_nontemporal_store(u0, d0);
      __builtin_nontemporal_store(u1, d1);
    } else {
      *d0 = u0;
      *d1 = u1;
    }
  }
}

template <typename T>
void launch_t(const RotaryArgs &a, int Dh, bool append, unsigned blocks, hipStream_t s) {
  if (Dh == 64) {
    if (append) hipLaunchKernelGGL((k_rotary<T, 64, true>), dim3(blocks), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_rotary<T, 64, false>), dim3(blocks), dim3(256), 0, s, a);
  } else {
    if (append) hipLaunchKernelGGL((k_rotary<T, 128, true>), dim3(blocks), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_rotary<T, 128, false>), dim3(blocks), dim3(256), 0, s, a);
  }
}

}  // namespace

namespace last {

// Tokens of a block: as many as give its 256 threads about one item of 32
// bytes each (two when appending, where a block first looks its tokens' places
// up), if that leaves 4 blocks a compute unit; else one, its heads dealt to
// several blocks until there are about 2 a compute unit. In bf16, heads of 128:
//   132096 tokens, 28 + 4 heads     1 token 363 us, 2 380, 4 398
//   100000 tokens, 12 + 2 heads     1 token 180 us, 2 134, 4 160
//   appending 108000, 12 + 2 + 2    1 token 304 us, 2 190, 4 154, 8 164
//   appending 16384, 28 + 4 + 4     1 token  68 us, 2  59, 4  61
static void shape(RotaryArgs *a, int items, bool append, int cus, int64_t *blocks) {
  const int heads = a->Hq + (append ? 2 : 1) * a->Hkv;
  const int want = std::max(1, std::min(kTokens, (2 * (append ? 512 : 256) + heads * items) / (2 * heads * items)));
  a->tokens = (int64_t)a->T * a->G >= (int64_t)want * 4 * cus ? want : 1;
  const int64_t b = ((int64_t)a->T + a->tokens - 1) / a->tokens * a->G;
  int64_t parts = std::max<int64_t>(1, (2 * cus) / b);
  a->parts = (int32_t)std::min<int64_t>(parts, std::max(1, heads / 8));
  *blocks = b * a->parts;
}

static int row_items(last_dtype dtype, int32_t Dh) { return Dh / (dtype == LAST_BF16 ? 16 : 8); }

int64_t rotary_blocks(RotaryArgs a, last_dtype dtype, int32_t Dh, bool append) {
  int64_t blocks = 0;
  shape(&a, row_items(dtype, Dh), append, device_cus(), &blocks);
  return blocks;
}

hipError_t launch_rotary(RotaryArgs a, last_dtype dtype, int32_t Dh, bool append, hipStream_t s) {
  int64_t blocks = 0;
  shape(&a, row_items(dtype, Dh), append, device_cus(), &blocks);
  launch_begin(append ? "rotary_append" : "rotary", s);
  if (dtype == LAST_F32) launch_t<float>(a, Dh, append, (unsigned)blocks, s);
  else launch_t<__bf16>(a, Dh, append, (unsigned)blocks, s);
  return launch_end(s);
}

}  // namespace last
