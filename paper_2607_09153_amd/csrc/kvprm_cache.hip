// The cache's traffic outside scoring for gfx950: rotary positions of queries and keys (k_rotary),
// rows of keys and values written into the paged cache (k_write_kv) and read back (k_read_kv).
#include <hip/hip_runtime.h>
#include <math.h>

#include "kvprm_internal.h"
#include "kvprm_mx_common.h"

namespace kvprm {

// ------------------------------------------------------------------------------- rotary

struct RotaryPart {
  const char *src;
  char *dst;
  int64_t ss, ds;  // row strides in elements
};
struct RotaryArgs {
  RotaryPart p[2];
  int heads0, heads;      // heads of the first tensor, of both
  int d, half, nrot;      // nrot: units of a head that are rotated
  int units;              // units per head
  uint32_t uinv, hinv;    // ceil(2^32 / units), ceil(2^32 / heads)
  int64_t rows;
  int rpb;                // rows per block
  const int32_t *pos;
  float mag, smag;        // factor on cosines and sines (the sines' negated for the transpose)
  double turn[kMaxRotaryPairs];  // turns per position of each pair
};

// 16 bytes that a call reads once, past the caches where it moves more than they hold.
__device__ __forceinline__ uint4 load_group(const uint4 *p, bool once) { return once ? ld_stream(p) : *p; }

// A vector of V elements of T, widened and back (rounded to nearest even). (bf16: one store of a native vector type.
// The compiler splits those of a struct of four words between branches that end alike, into 4 and 12 bytes: 22.5 us
// instead of 21.1 for k_rotary's 8192 rows.)
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
template <typename T, int V>
struct Vec;
template <>
struct Vec<float, 4> {
  static __device__ __forceinline__ void load(const float *p, float *v) {
    const float4 x = *(const float4 *)p;
    v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
  }
  static __device__ __forceinline__ void store(float *p, const float *v) {
    *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
  }
};
template <>
struct Vec<float, 1> {
  static __device__ __forceinline__ void load(const float *p, float *v) { v[0] = *p; }
  static __device__ __forceinline__ void store(float *p, const float *v) { *p = v[0]; }
};
__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
  typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
  typedef float f32x2v __attribute__((ext_vector_type(2)));
  const f32x2v x = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2v));
}
template <>
struct Vec<uint16_t, 8> {
  static __device__ __forceinline__ void load(const uint16_t *p, float *v) {
    const uint4 x = *(const uint4 *)p;
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ void store(uint16_t *p, const float *v) {
    *(u32x4v *)p = u32x4v{bf16x2(v[0], v[1]), bf16x2(v[2], v[3]), bf16x2(v[4], v[5]), bf16x2(v[6], v[7])};
  }
};
template <>
struct Vec<uint16_t, 1> {
  static __device__ __forceinline__ void load(const uint16_t *p, float *v) {
    v[0] = __uint_as_float((uint32_t)*p << 16);
  }
  static __device__ __forceinline__ void store(uint16_t *p, const float *v) {
    *p = (uint16_t)bf16x2(v[0], 0.f);
  }
};

// (a, b) -> m R(p f) (a, b) for every pair of the first 2 half dims of each head; the others are
// copied. Bound by memory. A block takes rpb rows: it first forms the cosine and sine of every
// (row, pair) in LDS, once for all heads, then walks the rows' units: V elements of a pair's first
// halves and the V matching ones (HALF), or V adjacent elements (INTERLEAVED), or V elements past
// the rotated ones. The angle's turns are reduced in 64 bits, p * f - round(p * f), since p f reaches
// 10^5 turns and more; the rest, at most half a turn, is exact enough in 32.
// V = 16 bytes where widths, strides and addresses allow, else one element.
// 16 heads of queries and 8 of keys of 128 dims, bf16, 8192 rows (100 MB moved): 21.1 us, 4.8 TB/s. Stores stay
// ordinary: non-temporal ones take less here (21.3 instead of 25.0 us where the rows come from memory, fp32 20.2
// instead of 23.4) and give it back where the rows are read next: a call and a copy of its result 47.0 instead of 43.5
// us at 48 MB written, 62.4 and 57.2 at 64, 85 and 93 at 96, 218 and 212 at 256 (bf16; fp32 alike). Two or four
// units of a thread in flight, loaded before the table is formed: 5 to 8% slower. 4093 rows of 36 heads of 64, fp32,
// adjacent pairs (75 MB): 14.1 us, partly from the caches, and 20 from memory (3.8 TB/s). One row for each of 16
// sequences: 7.6 us, the launch.
template <typename T, int V, bool HALF>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a) {
  __shared__ float2 cs[kRotaryCs];
  const int64_t row0 = (int64_t)blockIdx.x * a.rpb;
  const int nr = (int)min((int64_t)a.rpb, a.rows - row0);
  for (int i = threadIdx.x; i < nr * a.half; i += 256) {
    const int r = i / a.half, pair = i - r * a.half;
    const double t = (double)a.pos[row0 + r] * a.turn[pair];
    const float rest = (float)(t - rint(t));
    float s, c;
    sincospif(2.f * rest, &s, &c);
    cs[i] = make_float2(c * a.mag, s * a.smag);
  }
  __syncthreads();
  const uint32_t n = (uint32_t)nr * a.heads * a.units;
  for (uint32_t i = threadIdx.x; i < n; i += 256) {
    // (row, head), unit; the divisors' inverses are 0 for 1
    const uint32_t hr = a.uinv ? __umulhi(i, a.uinv) : i, u = i - hr * a.units;
    const uint32_t r = a.hinv ? __umulhi(hr, a.hinv) : hr, h = hr - r * a.heads;
    const bool second = (int)h >= a.heads0;
    const RotaryPart p = second ? a.p[1] : a.p[0];
    const int64_t at = (row0 + r);
    const int hh = (int)h - (second ? a.heads0 : 0);
    const T *src = (const T *)p.src + at * p.ss + (int64_t)hh * a.d;
    T *dst = (T *)p.dst + at * p.ds + (int64_t)hh * a.d;
    const float2 *c = cs + r * a.half;
    if ((int)u >= a.nrot) {  // kept dims
      const int e = 2 * a.half + ((int)u - a.nrot) * V;
      float x[V];
      Vec<T, V>::load(src + e, x);
      Vec<T, V>::store(dst + e, x);
    } else if (HALF) {
      const int e = (int)u * V;
      float x[V], y[V];
      Vec<T, V>::load(src + e, x);
      Vec<T, V>::load(src + a.half + e, y);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float2 w = c[e + k];
        const float xa = x[k], xb = y[k];
        x[k] = xa * w.x - xb * w.y;
        y[k] = xb * w.x + xa * w.y;
      }
      Vec<T, V>::store(dst + e, x);
      Vec<T, V>::store(dst + a.half + e, y);
    } else {
      // (one element at a time: a unit is a pair)
      constexpr int W = V == 1 ? 2 : V;
      const int e = (int)u * W;
      float x[W];
      if (V == 1) {
        Vec<T, 1>::load(src + e, x);
        Vec<T, 1>::load(src + e + 1, x + 1);
      } else {
        Vec<T, V>::load(src + e, x);
      }
#pragma unroll
      for (int k = 0; k < W; k += 2) {
        const float2 w = c[(e + k) >> 1];
        const float xa = x[k], xb = x[k + 1];
        x[k] = xa * w.x - xb * w.y;
        x[k + 1] = xb * w.x + xa * w.y;
      }
      if (V == 1) {
        Vec<T, 1>::store(dst + e, x);
        Vec<T, 1>::store(dst + e + 1, x + 1);
      } else {
        Vec<T, V>::store(dst + e, x);
      }
    }
  }
}

hipError_t launch_rotary(const kvprm_rope &rp, const double *turn, bool bf16, int64_t rows,
                         const int32_t *pos, const kvprm_rope_heads *parts, int num_parts,
                         bool transpose, hipStream_t s) {
  RotaryArgs a;
  const int eb = bf16 ? 2 : 4, v = 16 / eb;
  bool wide = true;
  a.heads = 0;
  a.heads0 = parts[0].heads;
  for (int i = 0; i < 2; ++i) {
    const kvprm_rope_heads &q = parts[i < num_parts ? i : 0];
    a.p[i] = RotaryPart{(const char *)q.src, (char *)q.dst, q.src_stride, q.dst_stride};
    if (i < num_parts) a.heads += q.heads;
    wide = wide && (((uintptr_t)q.src | (uintptr_t)q.dst) & 15) == 0 && q.src_stride % v == 0 &&
           q.dst_stride % v == 0;
  }
  const bool half = rp.layout == KVPRM_ROPE_HALF;
  a.d = rp.head_dim;
  a.half = rp.rotary_dim / 2;
  wide = wide && a.d % v == 0 && (half ? a.half : rp.rotary_dim) % v == 0;
  const int V = wide ? v : 1;
  a.nrot = half || !wide ? a.half / (half ? V : 1) : rp.rotary_dim / V;
  a.units = a.nrot + (a.d - rp.rotary_dim) / V;
  a.uinv = (uint32_t)(((1ull << 32) + a.units - 1) / a.units);
  a.hinv = (uint32_t)(((1ull << 32) + a.heads - 1) / a.heads);
  a.mag = (float)rp.magnitude;
  a.smag = transpose ? -a.mag : a.mag;
  for (int i = 0; i < a.half; ++i) a.turn[i] = turn[i];
  // Rows per block: one while that leaves the chip unfilled, then enough for four units a thread,
  // within the table. (Limits of 256 to 4096 units were within 3% of each other on 8192 rows.)
  const int64_t per_row = (int64_t)a.heads * a.units;
  int64_t rpb = 1;
  while (rpb < 16 && rpb * 2 * a.half <= kRotaryCs && rows > rpb * 1024 && rpb * per_row < 1024)
    rpb *= 2;
  a.rpb = (int)rpb;
  const int64_t most = rpb << 23;  // rows of a launch: 2^31 threads
  for (int64_t r0 = 0; r0 < rows; r0 += most) {
    a.rows = min(most, rows - r0);
    a.pos = pos + r0;
    for (int i = 0; i < 2; ++i) {
      const kvprm_rope_heads &q = parts[i < num_parts ? i : 0];
      a.p[i].src = (const char *)q.src + r0 * q.src_stride * eb;
      a.p[i].dst = (char *)q.dst + r0 * q.dst_stride * eb;
    }
    const dim3 grid((unsigned)((a.rows + rpb - 1) / rpb));
#define KVPRM_ROT(T_, V_)                                                             \
  if (half) hipLaunchKernelGGL((k_rotary<T_, V_, true>), grid, dim3(256), 0, s, a);   \
  else hipLaunchKernelGGL((k_rotary<T_, V_, false>), grid, dim3(256), 0, s, a)
    if (bf16) {
      if (wide) { KVPRM_ROT(uint16_t, 8); }
      else { KVPRM_ROT(uint16_t, 1); }
    } else {
      if (wide) { KVPRM_ROT(float, 4); }
      else { KVPRM_ROT(float, 1); }
    }
  }
#undef KVPRM_ROT
  return hipGetLastError();
}

// ------------------------------------------------------------------------------- cache rows

struct RowArgs {
  char *kp, *vp;       // this layer's pools
  float *ksc, *vsc;    // this layer's fp8 scales (or null)
  int nkv, num_pages;
  const int32_t *page_table;
  int max_pages;
  const int32_t *lengths;
  char *k, *v;         // rows
  int64_t ks, vs;      // row strides in elements
  int64_t num_rows;
  const int32_t *start, *index, *first;
  int max_rows;
  bool once;           // read_kv: tiles read past the caches
};

// Exponent of the smallest power of two s with 448 s >= amax (448 = 1.75 * 2^8), from the bits of
// a finite amax >= 0: 2^(E - 135), or the next one where the significand exceeds 1.75.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t b = __float_as_uint(amax);
  return max((int)(b >> 23) - 135 + ((b & 0x7FFFFFu) > 0x600000u), kMinScaleExp);
}
// Exponent of the smallest power of two >= s (s a positive normal number).
__device__ __forceinline__ int ceil_exponent(float s) {
  const uint32_t b = __float_as_uint(s);
  return (int)((b >> 23) & 255) - 127 + ((b & 0x7FFFFFu) != 0);
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Four values to e4m3 codes (nearest even; NaN and infinities to NaN).
__device__ __forceinline__ uint32_t fp8x4(const float *x) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = fabsf(x[i]) < INFINITY ? x[i] : __builtin_nanf("");
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], w, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  return (uint32_t)w;
}

// How a wave holds a tile's rows while it moves between token-major and stored order: a lane takes VS = 16
// bytes / sizeof(S) consecutive dims (e0 ..) of runs of RL consecutive slots, NP runs. A V tile keeps 4
// slots of a dim together, so a run is (half of) what a dim's cell holds, and no single bytes move.
template <int D, typename S>
struct RowMap {
  static constexpr int VS = 16 / (int)sizeof(S), LPR = D / VS, G = 64 / LPR, NR = 16 / G;
  static constexpr int RL = NR < 4 ? NR : 4, NP = NR / RL;
  int e0, first;  // first dim, first slot of the first run
  __device__ __forceinline__ RowMap(int lane) {
    const int rg = lane / LPR;
    e0 = (lane - rg * LPR) * VS;
    first = RL * rg;  // runs of a lane lie RL G slots apart
  }
  __device__ __forceinline__ int slot(int p, int i) const { return first + p * RL * G + i; }
};

// Byte of element (slot s, dim m) in a stored tile kept in LDS, with 16 bytes of padding after each 256, which
// spreads the cells of one dim over the banks.
template <int EB, int D>
__device__ __forceinline__ int key_byte(int s, int m) {
  constexpr int X = 16 / EB;
  const int g = (m / X) * 16 + s;
  return (g + g / 16) * 16 + m % X * EB;
}
template <int EB, int D>
__device__ __forceinline__ int value_byte(int s, int m) {
  constexpr int R = 4 / EB;
  const int g = ((m / (16 * R)) * 4 + s / 4) * 16 + m % 16;
  return (g + g / 16) * 16 + ((m / 16) % R * 4 + s % 4) * EB;
}
template <int EB, int D>
constexpr int tile_groups() { return D * EB + D * EB / 16; }

// N = 1, 2 or 4 values -> the cache's type, in the low bytes of up to 16.
template <int KVT, int N>
__device__ __forceinline__ uint4 narrow(const float *x) {
  uint4 r = make_uint4(0, 0, 0, 0);
  if constexpr (KVT == 0) {
    r.x = __float_as_uint(x[0]);
    if (N > 1) r.y = __float_as_uint(x[1]);
    if (N > 2) r.z = __float_as_uint(x[2]), r.w = __float_as_uint(x[3]);
  } else if constexpr (KVT == 1) {
    r.x = bf16x2(x[0], N > 1 ? x[1] : 0.f);
    if (N > 2) r.y = bf16x2(x[2], x[3]);
  } else {
    const float y[4] = {x[0], N > 1 ? x[1] : 0.f, N > 2 ? x[2] : 0.f, N > 2 ? x[3] : 0.f};
    r.x = fp8x4(y);
  }
  return r;
}
template <int BYTES>
__device__ __forceinline__ void put(unsigned char *p, const uint4 &v) {
  if constexpr (BYTES == 16) *(uint4 *)p = v;
  if constexpr (BYTES == 8) *(uint2 *)p = make_uint2(v.x, v.y);
  if constexpr (BYTES == 4) *(uint32_t *)p = v.x;
  if constexpr (BYTES == 2) *(uint16_t *)p = (uint16_t)v.x;
}
template <int BYTES>
__device__ __forceinline__ uint4 get(const unsigned char *p) {
  if constexpr (BYTES == 16) return *(const uint4 *)p;
  if constexpr (BYTES == 8) {
    const uint2 v = *(const uint2 *)p;
    return make_uint4(v.x, v.y, 0, 0);
  }
  if constexpr (BYTES == 4) return make_uint4(*(const uint32_t *)p, 0, 0, 0);
  return make_uint4(*(const uint16_t *)p, 0, 0, 0);
}
// The reverse of narrow.
template <int KVT, int N>
__device__ __forceinline__ void widen(const uint4 &v, float scale, float *x) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if constexpr (KVT == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __uint_as_float(w[i]);
  } else if constexpr (KVT == 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  } else {
    const float y[4] = {__builtin_amdgcn_cvt_f32_fp8(v.x, 0), __builtin_amdgcn_cvt_f32_fp8(v.x, 1),
                        __builtin_amdgcn_cvt_f32_fp8(v.x, 2), __builtin_amdgcn_cvt_f32_fp8(v.x, 3)};
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = y[i] * scale;
  }
}

// Rows of one (page, kv-head, part) tile, one wave: the tile's new rows in registers (16 bytes of a
// row per lane and load), for fp8 their largest magnitude and the tile's scale, the codes through LDS into
// the stored order, 16 bytes per lane and store. Only groups of 16 bytes that hold a new slot (or an
// old one whose scale grew) are stored; those that also hold other slots are read first.
// Bound by memory on long prompts: 8 prompts of 16384 to 32768 rows, 4 kv-heads of 128 dims, bf16 into fp8
// (590 MB moved): 121 us, 4.9 TB/s. Non-temporal loads and stores: 123 us; one wave for a page's keys and
// values: 124. Single tokens of 16 sequences: 6.6 us, the launch.
template <int KVT, int D, typename S>
__global__ __launch_bounds__(256) void k_write_kv(RowArgs a) {
  constexpr int EB = KVT == 0 ? 4 : KVT == 1 ? 2 : 1;
  typedef RowMap<D, S> Map;
  constexpr int VS = Map::VS, RL = Map::RL, NP = Map::NP;
  __shared__ uint4 lds[4][tile_groups<EB, D>()];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int b = blockIdx.y;
  const int item = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + wave);
  const int per = 2 * a.nkv, slotpage = item / per, pj = item - slotpage * per;
  const bool part = pj >= a.nkv;
  const int j = part ? pj - a.nkv : pj;
  const int L = a.lengths[b], r0 = a.start[b];
  if (L < 0 || r0 < 0) return;
  // rows of this candidate: at most max_rows, and no further than the page table
  const int n = (int)min((int64_t)min(a.start[b + 1] - r0, a.max_rows), (int64_t)a.max_pages * kPage - L);
  const int page = L / kPage + slotpage;
  if (n <= 0 || page * kPage >= L + n) return;
  const int id = a.page_table[(size_t)b * a.max_pages + page];
  if (id < 0 || id >= a.num_pages) return;
  const S *rows = (const S *)(part ? a.v : a.k);
  const int64_t stride = part ? a.vs : a.ks;
  const size_t tile = (size_t)id * a.nkv + j;
  float *scp = KVT == 2 ? (part ? a.vsc : a.ksc) + tile : nullptr;
  const float before = KVT == 2 ? *scp : 1.f;

  const Map at(lane);
  uint4 raw[NP][RL];
  uint32_t news = 0;  // slots this lane loads that are new
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int i = 0; i < RL; ++i) {
      const int slot = at.slot(p, i), t = page * kPage + slot - L;
      bool ok = t >= 0 && t < n;
      int64_t row = 0;
      if (ok) {
        row = a.index ? a.index[r0 + t] : r0 + t;
        ok = row >= 0 && row < a.num_rows;
      }
      raw[p][i] = make_uint4(0, 0, 0, 0);
      if (ok) {
        raw[p][i] = *(const uint4 *)(rows + row * stride + (int64_t)j * D + at.e0);
        news |= 1u << slot;
      }
    }
  float x[NP][RL][VS];
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int i = 0; i < RL; ++i) Vec<S, VS>::load((const S *)&raw[p][i], x[p][i]);
#pragma unroll
  for (int off = Map::LPR; off < 64; off <<= 1) news |= __shfl_xor(news, off, 64);
  if (!news) return;
  const int old = max(0, min(kPage, L - page * kPage));  // slots before the new ones

  uint4 *out = (uint4 *)(part ? a.vp : a.kp) + tile * (D * EB);
  float ratio = 1.f;
  bool grew = false;
  if (KVT == 2) {
    float m = 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int i = 0; i < RL; ++i)
#pragma unroll
        for (int k = 0; k < VS; ++k) {
          const float y = fabsf(x[p][i][k]);
          m = fmaxf(m, y < INFINITY ? y : 0.f);
        }
    int e = scale_exponent(wmax(m));
    if (old > 0) e = max(e, ceil_exponent(before));
    e = min(e, 126);  // (new values need 2^120 at most; the inverse of 2^126 is a normal number)
    const float scale = exp2i(e), inv = exp2i(-e);
    if (old > 0 && scale != before) {
      grew = true;
      ratio = before * inv;
    }
    if (lane == 0 && scale != before) *scp = scale;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int i = 0; i < RL; ++i)
#pragma unroll
        for (int k = 0; k < VS; ++k) x[p][i][k] *= inv;
  }

  // the new slots' values in the cache's type, in the stored order
  unsigned char *tb = (unsigned char *)lds[wave];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    if (!part) {
#pragma unroll
      for (int i = 0; i < RL; ++i)
#pragma unroll
        for (int k = 0; k < VS; k += 4)
          put<4 * EB>(tb + key_byte<EB, D>(at.slot(p, i), at.e0 + k), narrow<KVT, 4>(x[p][i] + k));
    } else {
#pragma unroll
      for (int k = 0; k < VS; ++k) {
        float y[4];
#pragma unroll
        for (int i = 0; i < RL; ++i) y[i] = x[p][i][k];
        put<RL * EB>(tb + value_byte<EB, D>(at.slot(p, 0), at.e0 + k), narrow<KVT, RL>(y));
      }
    }
  }
  __builtin_amdgcn_wave_barrier();
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  const uint32_t olds = old >= 16 ? 0xFFFFu : (1u << old) - 1u;
  const uint32_t touched = news | (grew ? olds : 0u);
  // codes of old slots at the grown scale
  auto rescaled = [&](uint32_t w) {
    const float y[4] = {__builtin_amdgcn_cvt_f32_fp8(w, 0) * ratio, __builtin_amdgcn_cvt_f32_fp8(w, 1) * ratio,
                        __builtin_amdgcn_cvt_f32_fp8(w, 2) * ratio, __builtin_amdgcn_cvt_f32_fp8(w, 3) * ratio};
    return fp8x4(y);
  };
  // bytes of word `word` of a V group that belong to the slots of `bits` (4 of them)
  auto bytes = [&](uint32_t bits, int word) {
    uint32_t m = 0;
    if (EB == 4) m = bits >> word & 1 ? ~0u : 0u;
    if (EB == 2) m = (bits >> (2 * (word & 1)) & 1 ? 0xFFFFu : 0u) | (bits >> (2 * (word & 1) + 1) & 1 ? 0xFFFF0000u : 0u);
    if (EB == 1) m = (bits & 1) * 0xFFu | (bits >> 1 & 1) * 0xFF00u | (bits >> 2 & 1) * 0xFF0000u | (bits >> 3) * 0xFF000000u;
    return m;
  };
#pragma unroll
  for (int it = 0; it < D * EB / 64; ++it) {
    const int gi = it * 64 + lane;
    // the group's slots: one key's, or four values'
    const int s = part ? 4 * (gi >> 4 & 3) : gi & 15;
    const uint32_t bits = part ? 15u : 1u, tch = touched >> s & bits, nw = news >> s & bits;
    if (!tch) continue;
    uint4 w = ((const uint4 *)tb)[gi + gi / 16];
    if (nw != bits) {
      const uint4 h = out[gi];
      uint32_t hw[4] = {h.x, h.y, h.z, h.w}, ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t mo = part ? bytes(olds >> s & 15, e) : (olds >> s & 1 ? ~0u : 0u);
        const uint32_t mn = part ? bytes(nw, e) : 0u;
        uint32_t kept = hw[e];
        if (KVT == 2 && grew) kept = (kept & ~mo) | (rescaled(kept) & mo);
        ww[e] = (kept & ~mn) | (ww[e] & mn);
      }
      w = make_uint4(ww[0], ww[1], ww[2], ww[3]);
    }
    out[gi] = w;
  }
}

// The reverse: one wave per (page, kv-head, part) tile, its 16-byte groups through LDS, rows of the
// wanted positions out, 16 bytes per lane and store. Bound by memory: 16 fp8 caches of 8192 to 16384 tokens,
// 8 kv-heads of 128 dims, to bf16 (1.2 GB moved): 225 us, 5.4 TB/s. Stores stay ordinary: non-temporal ones take
// 5 to 25% less, which a copy of the rows behind the call pays back up to 128 MB (both took 45.3 us at 64 MB, and 51.0
// with them; 191 and 175 at 256, 703 and 703 at 1 GB).
template <int KVT, int D, typename S>
__global__ __launch_bounds__(256) void k_read_kv(RowArgs a) {
  constexpr int EB = KVT == 0 ? 4 : KVT == 1 ? 2 : 1;
  typedef RowMap<D, S> Map;
  constexpr int VS = Map::VS, RL = Map::RL, NP = Map::NP;
  __shared__ uint4 lds[4][tile_groups<EB, D>()];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int b = blockIdx.y;
  const int item = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + wave);
  const int parts = (a.k ? 1 : 0) + (a.v ? 1 : 0);
  const int per = parts * a.nkv, slotpage = item / per, pj = item - slotpage * per;
  const bool part = !a.k || pj >= a.nkv;
  const int j = pj >= a.nkv ? pj - a.nkv : pj;
  const int L = (int)min((int64_t)a.lengths[b], (int64_t)a.max_pages * kPage);
  const int r0 = a.start[b], n = min(a.start[b + 1] - r0, a.max_rows);
  const int p0 = a.first ? a.first[b] : 0;  // position of the first row
  const int from = max(p0, 0), to = (int)min((int64_t)L, (int64_t)p0 + n);
  const int page = from / kPage + slotpage;
  if (n <= 0 || from >= to || page * kPage >= to) return;
  const int id = a.page_table[(size_t)b * a.max_pages + page];
  if (id < 0 || id >= a.num_pages) return;
  const size_t tile = (size_t)id * a.nkv + j;
  const uint4 *in = (const uint4 *)(part ? a.vp : a.kp) + tile * (D * EB);
  const float scale = KVT == 2 ? (part ? a.vsc : a.ksc)[tile] : 1.f;
  uint4 raw[D * EB / 64];
#pragma unroll
  for (int it = 0; it < D * EB / 64; ++it) raw[it] = load_group(in + it * 64 + lane, a.once);
#pragma unroll
  for (int it = 0; it < D * EB / 64; ++it) {
    const int gi = it * 64 + lane;
    lds[wave][gi + gi / 16] = raw[it];
  }
  __builtin_amdgcn_wave_barrier();
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  const unsigned char *tb = (const unsigned char *)lds[wave];
  S *rows = (S *)(part ? a.v : a.k);
  const int64_t stride = part ? a.vs : a.ks;
  const Map at(lane);
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    float x[RL][VS];
    if (!part) {
#pragma unroll
      for (int i = 0; i < RL; ++i)
#pragma unroll
        for (int k = 0; k < VS; k += 4)
          widen<KVT, 4>(get<4 * EB>(tb + key_byte<EB, D>(at.slot(p, i), at.e0 + k)), scale, x[i] + k);
    } else {
#pragma unroll
      for (int k = 0; k < VS; ++k) {
        float y[4];
        widen<KVT, RL>(get<RL * EB>(tb + value_byte<EB, D>(at.slot(p, 0), at.e0 + k)), scale, y);
#pragma unroll
        for (int i = 0; i < RL; ++i) x[i][k] = y[i];
      }
    }
#pragma unroll
    for (int i = 0; i < RL; ++i) {
      const int pos = page * kPage + at.slot(p, i);
      const int64_t row = (int64_t)r0 + pos - p0;
      if (pos < from || pos >= to || row < 0 || row >= a.num_rows) continue;
      Vec<S, VS>::store(rows + row * stride + (int64_t)j * D + at.e0, x[i]);
    }
  }
}

// The tiles are read past the caches where the rows take this much: 128 MB of fp32 rows from fp32 tiles 51.1 us so and
// 55.6 through the caches, bf16 from bf16 51.0 and 54.9, bf16 from fp8 39.9 and 42.0, 512 MB 192, 192 and 148 instead of
// 207, 206 and 157. A smaller call leaves the tiles there for whoever reads them next (8 MB take 7.9 and 8.0 us).
constexpr int64_t kOnceBytes = (int64_t)128 << 20;

static RowArgs row_args(const Dims &dm, const kvprm_kv_cache &c, const kvprm_batch &b, int layer,
                        const kvprm_kv_rows &r) {
  const size_t tiles = (size_t)c.num_pages * dm.nkv;
  const size_t bytes = tiles * kPage * dm.d * (dm.kvdt == 0 ? 4 : dm.kvdt == 1 ? 2 : 1);
  RowArgs a;
  a.kp = (char *)c.k_pages + layer * bytes;
  a.vp = (char *)c.v_pages + layer * bytes;
  a.ksc = dm.kvdt == 2 ? (float *)c.k_scale + layer * tiles : nullptr;
  a.vsc = dm.kvdt == 2 ? (float *)c.v_scale + layer * tiles : nullptr;
  a.nkv = dm.nkv;
  a.num_pages = c.num_pages;
  a.page_table = b.page_table;
  a.max_pages = b.max_pages;
  a.lengths = b.lengths;
  a.k = (char *)r.k;
  a.v = (char *)r.v;
  a.ks = r.k_stride;
  a.vs = r.v_stride;
  a.num_rows = r.num_rows;
  a.start = r.start;
  a.index = r.index;
  a.first = nullptr;
  a.max_rows = min(r.max_rows, b.max_pages * kPage);
  a.once = false;
  return a;
}

// Pages that hold at most n consecutive tokens, wherever they start.
static int pages_of(int n) { return (n + 2 * kPage - 2) / kPage; }

#define KVPRM_ROWS_S(K_, T_, D_)                                                                  \
  if (bf16) hipLaunchKernelGGL((K_<T_, D_, uint16_t>), grid, dim3(256), 0, s, a);                 \
  else hipLaunchKernelGGL((K_<T_, D_, float>), grid, dim3(256), 0, s, a)
#define KVPRM_ROWS_D(K_, T_)                                                                      \
  if (dm.d == 64) { KVPRM_ROWS_S(K_, T_, 64); }                                                   \
  else { KVPRM_ROWS_S(K_, T_, 128); }
#define KVPRM_ROWS(K_)                                                                            \
  if (dm.kvdt == 0) { KVPRM_ROWS_D(K_, 0) }                                                       \
  else if (dm.kvdt == 1) { KVPRM_ROWS_D(K_, 1) }                                                  \
  else { KVPRM_ROWS_D(K_, 2) }

hipError_t launch_write_kv(const Dims &dm, const kvprm_kv_cache &c, const kvprm_batch &b, int layer,
                           const kvprm_kv_rows &r, hipStream_t s) {
  const RowArgs a = row_args(dm, c, b, layer, r);
  const bool bf16 = r.dtype == KVPRM_BF16;
  const int pages = min(pages_of(a.max_rows), b.max_pages);
  const dim3 grid((unsigned)(((int64_t)pages * 2 * dm.nkv + 3) / 4), b.batch);
  KVPRM_ROWS(k_write_kv)
  return hipGetLastError();
}

hipError_t launch_read_kv(const Dims &dm, const kvprm_kv_cache &c, const kvprm_batch &b, int layer,
                          const kvprm_kv_rows &r, const int32_t *first, hipStream_t s) {
  RowArgs a = row_args(dm, c, b, layer, r);
  a.first = first;
  const bool bf16 = r.dtype == KVPRM_BF16;
  const int parts = (r.k ? 1 : 0) + (r.v ? 1 : 0);
  const int most = a.max_rows;  // positions of a candidate that hold tokens
  a.max_rows = r.max_rows;      // (rows of positions below 0 come on top of them)
  const int64_t rows = min((int64_t)most * b.batch, r.num_rows);
  a.once = rows * dm.nkv * dm.d * parts * (bf16 ? 2 : 4) >= kOnceBytes;
  const int pages = min(pages_of(most), b.max_pages);
  const dim3 grid((unsigned)(((int64_t)pages * parts * dm.nkv + 3) / 4), b.batch);
  KVPRM_ROWS(k_read_kv)
  return hipGetLastError();
}

}  // namespace kvprm
