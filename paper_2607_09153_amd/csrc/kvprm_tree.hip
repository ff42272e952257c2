// Attention of drafted tokens over the paged cache for gfx950: k_tree (chunks of cached pages and
// the drafted keys, by sequence, kv-head and columns) and k_tree_merge (the chunks' join).
#include <hip/hip_runtime.h>
#include <math.h>

#include "kvprm_attn_common.h"
#include "kvprm_internal.h"
#include "kvprm_mx_common.h"

namespace kvprm {

struct TreeArgs {
  const char *kp, *vp;     // this layer's pools
  const float *ksc, *vsc;  // this layer's fp8 scales (or null)
  int nkv, g, nq, num_pages, B;
  const int32_t *page_table;
  int max_pages;
  const int32_t *lengths;
  const void *q, *k, *v;
  void *o;
  int64_t qs, ks, vs, os;  // row strides in elements
  int64_t num_rows;
  const int32_t *start;
  int max_rows;
  const uint32_t *mask;
  int mask_words;
  uint32_t ginv;           // ceil(2^18 / g): c / g = (c * ginv) >> 18 for c < 4096 + 64, g <= 16
  int chunk_pages;         // cached pages of a chunk (a multiple of 2 kTreeWaves)
  int chunks;              // chunks of the grid: a candidate has no more
  int slots;               // chunk slots of a (row, q-head) in the workspace (at least chunks)
  float *pacc;             // [row][q-head][slot][D] chunk sums
  float2 *pml;             // [row][q-head][slot] chunk maximum (log2 units) and sum
};

constexpr int kTreeWaves = 4;
constexpr int kTreeSegStages = 128;  // page pairs whose ids (and scales) a k_tree_wide block holds at a time
constexpr int kTreeSeg = 64 * kTreeWaves;  // pages whose ids a block's lanes hold at a time

// The rows of one candidate, kept inside the arrays whatever `start` holds.
struct TreeRows {
  int L, n;    // cached tokens, drafted tokens
  int64_t r0;  // first row
};
__device__ __forceinline__ TreeRows tree_rows(const TreeArgs &a, int b) {
  TreeRows r;
  r.L = (int)max((int64_t)0, min((int64_t)a.lengths[b], (int64_t)a.max_pages * kPage));
  const int s0 = a.start[b], s1 = a.start[b + 1];
  r.r0 = s0;
  r.n = s0 < 0 || s0 >= a.num_rows ? 0 : (int)min((int64_t)min(s1 - s0, a.max_rows), a.num_rows - s0);
  return r;
}

// Chunks of a candidate with npages cached pages.
__device__ __forceinline__ int tree_chunks(const TreeArgs &a, int npages) {
  return max(1, min(a.chunks, (npages + a.chunk_pages - 1) / a.chunk_pages));
}

// The block's work: candidate, kv-head, chunk of its cached pages and block of its columns. The grid is
// one-dimensional and holds the blocks that exist, candidate by candidate (a scan over the lanes finds the
// candidate), then blocks without work, which leave at once: a grid of (chunk, column block, candidate) sides
// leaves them in a pattern that keeps part of the compute units idle on ragged batches. Blocks go to the
// eight XCDs in turn; the column blocks of one chunk, which read the same pages, lie eight apart, so
// that they share an L2.
struct TreeItem {
  int b, j, chunk, colblock;
};
__device__ __forceinline__ bool tree_item(const TreeArgs &a, int cols_per_block, TreeItem &it) {
  const int lane = threadIdx.x & 63;
  int id = blockIdx.x;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    int items_l = 0, cb_l = 0;
    if (b0 + lane < a.B) {
      const TreeRows r = tree_rows(a, b0 + lane);
      if (r.n > 0) {
        items_l = tree_chunks(a, (r.L + kPage - 1) / kPage) * a.nkv;
        cb_l = (r.n * a.g + cols_per_block - 1) / cols_per_block;
      }
    }
    const int n_l = items_l * cb_l, cum_l = lane_scan(n_l);
    const int total = __builtin_amdgcn_readlane(cum_l, 63);
    if (id >= total) {
      id -= total;
      continue;
    }
    const int k = __builtin_popcountll(__ballot(id >= cum_l));
    const int items = lane_value(items_l, k), cb = lane_value(cb_l, k);
    id -= lane_value(cum_l, k) - items * cb;
    const int full = items & ~7;  // items in groups of eight
    int item;
    if (id < full * cb) {
      const int grp = id / (8 * cb), rem = id - grp * 8 * cb;
      it.colblock = rem >> 3;
      item = grp * 8 + (rem & 7);
    } else {
      const int rem = id - full * cb, last = items - full;
      it.colblock = rem / last;
      item = full + rem - it.colblock * last;
    }
    it.b = b0 + k;
    it.chunk = item / a.nkv;
    it.j = item - it.chunk * a.nkv;
    return true;
  }
  return false;
}

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void load4(const float *p, float *v) {
  const float4 x = *(const float4 *)p;
  v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
}
__device__ __forceinline__ void load4(const uint16_t *p, float *v) {
  const uint2 x = *(const uint2 *)p;
  v[0] = __uint_as_float(x.x << 16), v[1] = __uint_as_float(x.x & 0xFFFF0000u);
  v[2] = __uint_as_float(x.y << 16), v[3] = __uint_as_float(x.y & 0xFFFF0000u);
}
__device__ __forceinline__ void store4(float *p, const float *v) {
  *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store4(uint16_t *p, const float *v) {
  typedef __bf16 bf16x4v __attribute__((ext_vector_type(4)));
  typedef float f32x4v __attribute__((ext_vector_type(4)));
  const f32x4v x = {v[0], v[1], v[2], v[3]};
  *(uint2 *)p = __builtin_bit_cast(uint2, __builtin_convertvector(x, bf16x4v));
}

// The running softmax of a wave's columns: one column per lane % 16 and column tile, the four lanes
// of a column hold the same m (log2 units), their own tokens' share of l, and 4 of each 16 output
// dims: acc[nb][i] = dim 16 nb + 4 (lane / 16) + i.
template <int D>
struct Soft {
  float m, l;
  floatx4 acc[D / 16];
  __device__ __forceinline__ void init() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  // N scores of this lane (log2 units, -inf where masked) -> their weights; the state moves to the
  // new maximum first.
  template <int N>
  __device__ __forceinline__ void weights(float (&s)[N]) {
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < N; ++i) mx = fmaxf(mx, s[i]);
    const float mn = fmaxf(m, column_max(mx));
    if (__any(mn > m)) {
      const float alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] *= alpha;
    }
    const float ms = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s[i] = __builtin_amdgcn_exp2f(s[i] - ms);
      l += s[i];
    }
  }
};

// One step over 16 tokens with every operand in fp32: scores of the lane's tokens 4 (lane / 16) + i
// from kf and qf (dims 16 kk + 4 (lane / 16) + e at 4 kk + e, of token or column lane % 16), softmax,
// acc += vf^T p (vf[nb][i]: dim 16 nb + lane % 16 of token 4 (lane / 16) + i). ok: tokens attended to.
template <int D>
__device__ __forceinline__ void step32(const float (&kf)[D / 4], const float (&vf)[D / 16][4],
                                       const float (&qf)[D / 4], const bool (&ok)[4], float rs,
                                       Soft<D> &st, float (&p)[4]) {
  floatx4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < D / 4; i += 2) {
    s0 = mfma4(kf[i], qf[i], s0);
    s1 = mfma4(kf[i + 1], qf[i + 1], s1);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = ok[i] ? (s0[i] + s1[i]) * rs : -INFINITY;
  st.template weights<4>(p);
#pragma unroll
  for (int nb = 0; nb < D / 16; ++nb)
#pragma unroll
    for (int i = 0; i < 4; ++i) st.acc[nb] = mfma4(vf[nb][i], p[i], st.acc[nb]);
}

// One column's query in fp32, in step32's order.
template <int D, typename T>
__device__ __forceinline__ void query32(const T *q, int cq, bool present, float (&qf)[D / 4]) {
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    float v[4];
    load4(q + 16 * kk + 4 * cq, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) qf[4 * kk + e] = present ? v[e] : 0.f;
  }
}

// Terms of fp32 operands in bf16: rows in bf16 are one term, fp32 rows three (24 bits); the
// weights, in (0, 1], enter as two terms (16 bits) for bf16 results, whose own rounding is at 2^-9,
// and three for fp32 ones. One term would add an error the size of the bf16 result's rounding.
template <typename T>
struct Terms;
template <>
struct Terms<uint16_t> {
  static constexpr int Q = 1, P = 2;
};
template <>
struct Terms<float> {
  static constexpr int Q = 3, P = 3;
};

// o = softmax(q K^T / sqrt(d)) V for NC tiles of 16 columns (drafted token, q-head of the kv-head's
// group), over one chunk of a candidate's cached pages; the last chunk also takes the drafted keys.
// A block's four waves take page pairs in turn and join their softmax states in LDS, so that a chunk is
// one partial result.
// A page pair (32 tokens) is one step: S = K Q^T, a running softmax in registers, O^T += V^T P^T, all
// on the matrix cores with the cache's tiles as they lie in memory (see kvprm_attn.hip).
template <int KVT, int D, int NC, typename T>
__global__ __launch_bounds__(64 * kTreeWaves) void k_tree(TreeArgs a) {
  constexpr int NKB = D / 32, NDB = D / 16, W = kTreeWaves;
  constexpr int QT = Terms<T>::Q, PT = Terms<T>::P;
  constexpr size_t TILE = (size_t)kPage * D * (KVT == 0 ? 4 : KVT == 1 ? 2 : 1);
  __shared__ floatx4 sacc[W][NC][NDB][64];
  __shared__ float2 sml[W][NC * 16];
  TreeItem it;
  if (!tree_item(a, 16 * NC, it)) return;
  const int b = it.b, j = it.j, c = it.chunk;
  const TreeRows tr = tree_rows(a, b);
  const int L = tr.L, n = tr.n, g = a.g;
  const int cols = n * g, col0 = it.colblock * 16 * NC;
  const int npages = (L + kPage - 1) / kPage, nc = tree_chunks(a, npages);
  const int p0 = c * a.chunk_pages, np = min(a.chunk_pages, npages - p0);
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, cn = lane & 15, cq = lane >> 4;
  const float rs = kLog2e / sqrtf((float)D);

  // this lane's columns: drafted token and q-head
  int tok[NC], head[NC];
  bool present[NC];
#pragma unroll
  for (int ct = 0; ct < NC; ++ct) {
    const int col = col0 + ct * 16 + cn;
    present[ct] = col < cols;
    tok[ct] = present[ct] ? (int)(((uint32_t)col * a.ginv) >> 18) : 0;
    head[ct] = j * g + (present[ct] ? col - tok[ct] * g : 0);
  }
  auto qrow = [&](int ct) { return (const T *)a.q + (tr.r0 + tok[ct]) * a.qs + (int64_t)head[ct] * D; };
  Soft<D> st[NC];
#pragma unroll
  for (int ct = 0; ct < NC; ++ct) st[ct].init();

  for (int seg = 0; seg < np; seg += kTreeSeg) {
    const int sp = p0 + seg, sn = min(kTreeSeg, np - seg);  // pages of this segment
    if constexpr (KVT == 0) {
      // wave w takes pages w, w + W, ...; lane i holds the id of its i-th page
      const int mine = (sn - w + W - 1) / W;
      if (mine <= 0) continue;
      const int id_l =
          min(max(a.page_table[(size_t)b * a.max_pages + sp + min(w + W * lane, sn - 1)], 0), a.num_pages - 1);
      float qf[NC][D / 4];
#pragma unroll
      for (int ct = 0; ct < NC; ++ct) query32<D>(qrow(ct), cq, present[ct], qf[ct]);
      for (int i = 0; i < mine; ++i) {
        const size_t tile = ((size_t)lane_value(id_l, i) * a.nkv + j) * TILE;
        const float4 *kt = (const float4 *)(a.kp + tile), *vt = (const float4 *)(a.vp + tile);
        const int t0 = (sp + w + W * i) * kPage + 4 * cq;
        bool ok[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) ok[e] = t0 + e < L;
        float kf[D / 4], vf[NDB][4];
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          load4((const float *)(kt + (4 * kk + cq) * 16 + cn), kf + 4 * kk);
          load4((const float *)(vt + kk * 64 + lane), vf[kk]);
          // K: the tile's 4-dim block 4 kk + cq of slot cn; V: slots 4 cq.. of dim 16 kk + cn
#pragma unroll
          for (int e = 0; e < 4; ++e) vf[kk][e] = ok[e] ? vf[kk][e] : 0.f;
        }
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
          float p[4];
          step32<D>(kf, vf, qf[ct], ok, rs, st[ct], p);
        }
      }
    } else {
      // wave w takes page pairs w, w + W, ...; lanes 2i and 2i + 1 hold its i-th pair's ids
      const int pairs = (sn + 1) >> 1, mine = (pairs - w + W - 1) / W;
      if (mine <= 0) continue;
      const int pg = min(2 * (w + W * (lane >> 1)) + (lane & 1), sn - 1);
      const int id_l = min(max(a.page_table[(size_t)b * a.max_pages + sp + pg], 0), a.num_pages - 1);
      float ksc_l = 0.f, vsc_l = 0.f;
      if (KVT == 2) {
        ksc_l = a.ksc[(size_t)id_l * a.nkv + j];
        vsc_l = a.vsc[(size_t)id_l * a.nkv + j];
      }
      auto load_pair = [&](int i, PairRaw<D> &r) {
        const int ia = 2 * min(i, mine - 1);
        const size_t ta = ((size_t)lane_value(id_l, ia) * a.nkv + j) * TILE;
        const size_t tb = ((size_t)lane_value(id_l, ia + 1) * a.nkv + j) * TILE;
        load_pair_raw<KVT, D, false>((const uint4 *)(a.kp + ta), (const uint4 *)(a.kp + tb),
                                     (const uint4 *)(a.vp + ta), (const uint4 *)(a.vp + tb), lane, r);
      };
      PairRaw<D> r0, r1;
      load_pair(0, r0);
      uint4 qo[NC][QT][NKB];
#pragma unroll
      for (int ct = 0; ct < NC; ++ct) {
        const T *qr = qrow(ct);
#pragma unroll
        for (int kk = 0; kk < NKB; ++kk) {
          const int dim = KVT == 1 ? kk * 32 + 8 * cq : 16 * (4 * (kk >> 1) + cq) + 8 * (kk & 1);
          if constexpr (QT == 1) {
            const uint4 v = *(const uint4 *)(qr + dim);
            qo[ct][0][kk] = present[ct] ? v : make_uint4(0, 0, 0, 0);
          } else {
            float v[8];
            load4((const float *)qr + dim, v);
            load4((const float *)qr + dim + 4, v + 4);
            uint32_t t[3][4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              split3(present[ct] ? v[2 * e] : 0.f, present[ct] ? v[2 * e + 1] : 0.f, t[0][e], t[1][e], t[2][e]);
#pragma unroll
            for (int x = 0; x < QT; ++x) qo[ct][x][kk] = make_uint4(t[x][0], t[x][1], t[x][2], t[x][3]);
          }
        }
      }
      auto compute = [&](int i, const PairRaw<D> &r) {
        uint4 KA[NKB], KB[NKB];
        uint2 VA[NDB], VB[NDB];
        unpack_pair<KVT, D>(r, KA, KB, VA, VB);
        const int la = 2 * i;
        const float sca = KVT == 2 ? lane_value(ksc_l, la) * rs : rs;
        const float scb = KVT == 2 ? lane_value(ksc_l, la + 1) * rs : rs;
        const int t0 = (sp + 2 * (w + W * i)) * kPage;
        const bool tail = t0 + 2 * kPage > L;  // slots at or past L in this pair (they may hold anything)
        const int left = L - t0 - 4 * cq;      // this lane's tokens: 0..3 of page A, 16..19 of page B
        if (tail) {
          const uint32_t a0 = (left > 0 ? 0xFFFFu : 0u) | (left > 1 ? 0xFFFF0000u : 0u);
          const uint32_t a1 = (left > 2 ? 0xFFFFu : 0u) | (left > 3 ? 0xFFFF0000u : 0u);
          const uint32_t b0 = (left > 16 ? 0xFFFFu : 0u) | (left > 17 ? 0xFFFF0000u : 0u);
          const uint32_t b1 = (left > 18 ? 0xFFFFu : 0u) | (left > 19 ? 0xFFFF0000u : 0u);
#pragma unroll
          for (int nb = 0; nb < NDB; ++nb) {
            VA[nb].x &= a0, VA[nb].y &= a1;
            VB[nb].x &= b0, VB[nb].y &= b1;
          }
        }
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
          floatx4 sa = {0.f, 0.f, 0.f, 0.f}, sb = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kk = 0; kk < NKB; ++kk)
#pragma unroll
            for (int x = 0; x < QT; ++x) {
              sa = mfma16(KA[kk], qo[ct][x][kk], sa);
              sb = mfma16(KB[kk], qo[ct][x][kk], sb);
            }
          float p[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = sa[e] * sca;
            p[4 + e] = sb[e] * scb;
          }
          if (tail) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              p[e] = left > e ? p[e] : -INFINITY;
              p[4 + e] = left > 16 + e ? p[4 + e] : -INFINITY;
            }
          }
          st[ct].template weights<8>(p);
          if (KVT == 2) {
            const float vsa = lane_value(vsc_l, la), vsb = lane_value(vsc_l, la + 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              p[e] *= vsa;
              p[4 + e] *= vsb;
            }
            if (tail) {  // (the scale of a page past the last, repeated, times 0)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                p[e] = left > e ? p[e] : 0.f;
                p[4 + e] = left > 16 + e ? p[4 + e] : 0.f;
              }
            }
          }
          uint32_t t[3][4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (PT == 2) split2(p[2 * e], p[2 * e + 1], t[0][e], t[1][e]);
            else split3(p[2 * e], p[2 * e + 1], t[0][e], t[1][e], t[2][e]);
          }
#pragma unroll
          for (int nb = 0; nb < NDB; ++nb) {
            const uint4 vo = make_uint4(VA[nb].x, VA[nb].y, VB[nb].x, VB[nb].y);
#pragma unroll
            for (int x = 0; x < PT; ++x)
              st[ct].acc[nb] = mfma16(vo, make_uint4(t[x][0], t[x][1], t[x][2], t[x][3]), st[ct].acc[nb]);
          }
        }
      };
      for (int i = 0; i < mine; i += 2) {
        load_pair(i + 1, r1);
        __builtin_amdgcn_sched_barrier(0);
        compute(i, r0);
        __builtin_amdgcn_sched_barrier(0);
        load_pair(i + 2, r0);
        __builtin_amdgcn_sched_barrier(0);
        if (i + 1 < mine) compute(i + 1, r1);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

  // the drafted keys, 16 at a time, in fp32 (T^2 products beside T L: the fp32 matrix instructions
  // need no split); wave w takes tiles w, w + W, ...
  if (c == nc - 1) {
    const T *kd = (const T *)a.k + tr.r0 * a.ks + (int64_t)j * D;
    const T *vd = (const T *)a.v + tr.r0 * a.vs + (int64_t)j * D;
    for (int t0 = 16 * w; t0 < n; t0 += 16 * W) {
      float kf[D / 4], vf[NDB][4];
      const T *kr = kd + (int64_t)min(t0 + cn, n - 1) * a.ks;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) load4(kr + 16 * kk + 4 * cq, kf + 4 * kk);
      bool bad = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const T *vr = vd + (int64_t)min(t0 + 4 * cq + e, n - 1) * a.vs;
#pragma unroll
        for (int nb = 0; nb < NDB; ++nb) {
          vf[nb][e] = widen(vr[16 * nb + cn]);
          bad = bad || !(fabsf(vf[nb][e]) < INFINITY);
        }
      }
      // Infinities and NaN among the values: 0 times them would reach the columns that do not attend
      // to them, so they leave the product and are added column by column.
      const bool any_bad = __any(bad);
      if (any_bad) {
#pragma unroll
        for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) vf[nb][e] = fabsf(vf[nb][e]) < INFINITY ? vf[nb][e] : 0.f;
      }
#pragma unroll
      for (int ct = 0; ct < NC; ++ct) {
        float qf[D / 4], p[4];
        query32<D>(qrow(ct), cq, present[ct], qf);
        bool ok[4];
        uint32_t bits = 0;
        if (a.mask) bits = a.mask[(tr.r0 + tok[ct]) * a.mask_words + (t0 >> 5)] >> (t0 & 31);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = t0 + 4 * cq + e;
          ok[e] = t < n && (a.mask ? (bits >> (4 * cq + e) & 1) != 0 : t <= tok[ct]);
        }
        step32<D>(kf, vf, qf, ok, rs, st[ct], p);
        if (any_bad) {
          for (int t = 0; t < 16 && t0 + t < n; ++t) {
            // the weight of token t for this lane's column, from the lane that holds it
            float pt = 0.f;
            bool okt = false;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if ((t & 3) == e) pt = p[e], okt = ok[e];
            pt = __shfl(pt, (t >> 2) * 16 + cn, 64);
            okt = __shfl((int)okt, (t >> 2) * 16 + cn, 64) != 0;
#pragma unroll
            for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float v = widen(vd[(int64_t)(t0 + t) * a.vs + 16 * nb + 4 * cq + e]);
                if (okt && !(fabsf(v) < INFINITY)) st[ct].acc[nb][e] += pt * v;
              }
          }
        }
      }
    }
  }

  // join the waves' states: each wave adds the output dims of its own share, in wave order
#pragma unroll
  for (int ct = 0; ct < NC; ++ct) {
    const float l = column_sum(st[ct].l);
    if (cq == 0) sml[w][ct * 16 + cn] = make_float2(st[ct].m, l);
#pragma unroll
    for (int nb = 0; nb < NDB; ++nb) sacc[w][ct][nb][lane] = st[ct].acc[nb];
  }
  __syncthreads();
#pragma unroll
  for (int ct = 0; ct < NC; ++ct) {
    float f[W], M = -INFINITY, l = 0.f;
#pragma unroll
    for (int x = 0; x < W; ++x) M = fmaxf(M, sml[x][ct * 16 + cn].x);
#pragma unroll
    for (int x = 0; x < W; ++x) {
      const float2 ml = sml[x][ct * 16 + cn];
      f[x] = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
      l += f[x] * ml.y;
    }
    const int64_t row = tr.r0 + tok[ct];
    const int64_t at = (row * a.nq + head[ct]) * a.slots + c;
#pragma unroll
    for (int k = 0; k < NDB / W; ++k) {
      const int nb = w * (NDB / W) + k;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < W; ++x) {
        const floatx4 y = sacc[x][ct][nb][lane];
        // (a wave that saw no token adds nothing)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += f[x] * y[e];
      }
      if (!present[ct]) continue;
      if (nc == 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = l == 0.f ? 0.f : v[e] / l;
        store4((T *)a.o + row * a.os + (int64_t)head[ct] * D + 16 * nb + 4 * cq, v);
      } else {
        store4(a.pacc + at * D + 16 * nb + 4 * cq, v);
      }
    }
    if (nc > 1 && w == 0 && cq == 0 && present[ct]) a.pml[at] = make_float2(M, l);
  }
}

// ------------------------------------------------------------------------------- wide drafts

typedef float floatx16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ floatx16 mfma32(const uint4 &a, const uint4 &b, const floatx16 &c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The same for drafts of many columns (bf16 rows): here the waves share the pages and split the
// columns, 32 each. A stage is a page pair (32 tokens) in LDS as bf16 tiles in the stored order (fp8
// tiles are widened on their way, exactly), double buffered, the next pair's loads in flight while one is
// computed. 32x32x16 products: S = K Q^T (a lane holds tokens 8 i + 4 h + e, h = lane / 32, of
// column lane % 32), softmax, O^T += V^T P^T with P in two bf16 terms, tokens in S's order (8 slots 4 h..,
// 8 + 4 h.. of one page are one operand). The drafted keys are stages of their own behind the last
// chunk's pages, laid out as a page pair.
template <int KVT, int D, int W>
__global__ __launch_bounds__(64 * W, 2) void k_tree_wide(TreeArgs a) {
  typedef uint16_t T;
  constexpr int KS = D / 16, NT = D / 32, TC = 2 * D;  // k steps, output tiles, 16-byte groups of a bf16 tile
  constexpr int SC = KVT == 1 ? 2 * TC : TC;           // 16-byte groups of a pair in memory
  constexpr int NLC = (SC + 64 * W - 1) / (64 * W);    // of these per thread, K or V
  constexpr int SEG = kTreeSegStages;
  __shared__ uint4 kb[2][2 * TC], vb[2][2 * TC];
  __shared__ int id_s[2 * SEG];                        // page ids of a segment, and their scales
  __shared__ float ksc_s[KVT == 2 ? 2 * SEG : 1], vsc_s[KVT == 2 ? 2 * SEG : 1];
  __shared__ int bad_s;
  TreeItem it;
  if (!tree_item(a, 32 * W, it)) return;
  const int b = it.b, j = it.j, c = it.chunk;
  const TreeRows tr = tree_rows(a, b);
  const int L = tr.L, n = tr.n, g = a.g;
  const int npages = (L + kPage - 1) / kPage, nc = tree_chunks(a, npages);
  const int p0 = c * a.chunk_pages, np = min(a.chunk_pages, npages - p0);
  const int tid = threadIdx.x, lane = tid & 63, cn = lane & 31, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cols = n * g, col0 = it.colblock * 32 * W + w * 32, col = col0 + cn;
  const bool busy = col0 < cols, present = col < cols;
  const int tok = present ? (int)(((uint32_t)col * a.ginv) >> 18) : 0;
  const int head = j * g + (present ? col - tok * g : 0);
  const float rs = kLog2e / sqrtf((float)D);
  const int ncache = (np + 1) >> 1;                    // stages of cached pages
  const int nfull = max(0, L - p0 * kPage) >> 5;       // of these, the first without a slot at or past L
  const T *kd = (const T *)a.k + tr.r0 * a.ks + (int64_t)j * D;
  const T *vd = (const T *)a.v + tr.r0 * a.vs + (int64_t)j * D;

  uint4 qo[KS];
  {
    const T *q = (const T *)a.q + (tr.r0 + tok) * a.qs + (int64_t)head * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const uint4 v = *(const uint4 *)(q + 16 * ks + 8 * h);
      qo[ks] = present ? v : make_uint4(0, 0, 0, 0);
    }
  }
  // A stage's tiles in registers: 16-byte groups of K and V.
  struct Pair {
    uint4 k[NLC], v[NLC];
  };
  int s0 = 0, se = 0;  // the segment's stages
  // (no branch around the loads, which would join registers still in flight: stages past the end repeat
  // the last one)
  auto load_stage = [&](int s, Pair &r) {
    const int i = 2 * (min(s, se - 1) - s0);
    constexpr size_t TILE = (size_t)kPage * D * (KVT == 1 ? 2 : 1);
    const size_t ta = ((size_t)__builtin_amdgcn_readfirstlane(id_s[i]) * a.nkv + j) * TILE;
    const size_t tb = ((size_t)__builtin_amdgcn_readfirstlane(id_s[i + 1]) * a.nkv + j) * TILE;
#pragma unroll
    for (int k = 0; k < NLC; ++k) {
      // this wave's first group; pairs of fewer groups than threads are read twice
      const int i0 = (k * 64 * W + w * 64) % SC;
      const size_t t = i0 >= SC / 2 ? tb : ta;
      r.k[k] = ((const uint4 *)(a.kp + t))[i0 % (SC / 2) + lane];
      r.v[k] = ((const uint4 *)(a.vp + t))[i0 % (SC / 2) + lane];
    }
  };
  auto store_stage = [&](int s, const Pair &r) {
    if (s >= se) return;
    uint4 *kt = kb[s & 1], *vt = vb[s & 1];
    const int left = L - (p0 + 2 * s) * kPage;  // valid slots from the pair's first on
#pragma unroll
    for (int k = 0; k < NLC; ++k) {
      const int i0 = (k * 64 * W + w * 64) % SC;
      const bool second = i0 >= SC / 2;
      const int i = i0 % (SC / 2) + lane, at = second ? TC : 0;
      // slots at or past L may hold anything: as values they become zeros
      uint32_t m0 = ~0u, m1 = ~0u;
      if (left < 32) {
        const int q = left - (second ? 16 : 0) - 4 * ((i >> 4) & 3);
        m0 = (q > 0 ? 0xFFFFu : 0u) | (q > 1 ? 0xFFFF0000u : 0u);
        m1 = (q > 2 ? 0xFFFFu : 0u) | (q > 3 ? 0xFFFF0000u : 0u);
      }
      const uint4 rk = r.k[k], rv = r.v[k];
      if (KVT == 1) {
        kt[at + i] = rk;
        vt[at + i] = make_uint4(rv.x & m0, rv.y & m1, rv.z & m0, rv.w & m1);
      } else {
        // 16 dims of a slot -> two groups of 8; 4 dims of 4 slots -> two groups of 2
        uint4 *kp = kt + at + (i >> 4) * 32 + (i & 15);
        kp[0] = make_uint4(fp8x2_to_bf16x2<false>(rk.x), fp8x2_to_bf16x2<true>(rk.x),
                           fp8x2_to_bf16x2<false>(rk.y), fp8x2_to_bf16x2<true>(rk.y));
        kp[16] = make_uint4(fp8x2_to_bf16x2<false>(rk.z), fp8x2_to_bf16x2<true>(rk.z),
                            fp8x2_to_bf16x2<false>(rk.w), fp8x2_to_bf16x2<true>(rk.w));
        uint4 *vp = vt + at + (i >> 6) * 128 + (i & 63);
        vp[0] = make_uint4(fp8x2_to_bf16x2<false>(rv.x) & m0, fp8x2_to_bf16x2<true>(rv.x) & m1,
                           fp8x2_to_bf16x2<false>(rv.y) & m0, fp8x2_to_bf16x2<true>(rv.y) & m1);
        vp[64] = make_uint4(fp8x2_to_bf16x2<false>(rv.z) & m0, fp8x2_to_bf16x2<true>(rv.z) & m1,
                            fp8x2_to_bf16x2<false>(rv.w) & m0, fp8x2_to_bf16x2<true>(rv.w) & m1);
      }
    }
  };
  // 32 drafted tokens from t0 on as a page pair in buffer 0.
  auto store_draft = [&](int t0) {
    uint4 *kt = kb[0], *vt = vb[0];
    bool bad = false;
    for (int i = tid; i < 2 * TC; i += 64 * W) {
      const int t = i / (D / 8), e = 8 * (i % (D / 8)), at = (t >> 4) * TC, sl = t & 15;
      uint4 rk = make_uint4(0, 0, 0, 0), rv = rk;
      if (t0 + t < n) {
        rk = *(const uint4 *)(kd + (t0 + t) * a.ks + e);
        rv = *(const uint4 *)(vd + (t0 + t) * a.vs + e);
      }
      kt[at + (e >> 3) * 16 + sl] = rk;
      const uint32_t x[4] = {rv.x, rv.y, rv.z, rv.w};
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const int mm = e + y;
        uint32_t v = (x[y >> 1] >> (16 * (y & 1))) & 0xFFFFu;
        // infinities and NaN leave the product (see below)
        if ((v & 0x7F80u) == 0x7F80u) bad = true, v = 0;
        ((uint16_t *)(vt + at))[((((mm >> 5) * 4 + (sl >> 2)) * 16 + (mm & 15)) * 2 + ((mm >> 4) & 1)) * 4 + (sl & 3)] =
            (uint16_t)v;
      }
    }
    if (bad) bad_s = 1;
  };

  float m = -INFINITY, l = 0.f;
  floatx16 acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;

  // One stage, cached pages (d0 < 0) or the drafted tokens from d0 on; MASKED: only the tokens of `ok`
  // (bit r: this lane's r-th) count.
  auto compute = [&](int s, auto masked, uint32_t ok, int d0) {
    const int buf = d0 < 0 ? s & 1 : 0;
    const uint4 *kt = kb[buf] + (cn >> 4) * TC + h * 16 + (cn & 15);
    const uint4 *vt = vb[buf] + (cn >> 4) * 64 + h * 16 + (cn & 15);
    floatx16 sv;
#pragma unroll
    for (int e = 0; e < 16; ++e) sv[e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) sv = mfma32(kt[ks * 32], qo[ks], sv);
    float ka = rs, kc = rs, va = 1.f, vc = 1.f;
    if (KVT == 2 && d0 < 0) {
      const int i = 2 * (s - s0);
      ka = ksc_s[i] * rs, kc = ksc_s[i + 1] * rs, va = vsc_s[i], vc = vsc_s[i + 1];
    }
    if (decltype(masked)::value) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sv[e] = ok >> e & 1 ? sv[e] : -INFINITY;
    }
    float ma = sv[0], mb = sv[8];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
      ma = fmaxf(ma, sv[e]);
      mb = fmaxf(mb, sv[8 + e]);
    }
    float mx = fmaxf(ma * ka, mb * kc);  // (scales are positive; -inf stays -inf)
    {
      const uint32_t u = __float_as_uint(mx);
      const auto t = __builtin_amdgcn_permlane32_swap(u, u, false, false);
      mx = fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
    }
    const float mn = fmaxf(m, mx);
    if (__any(mn > m)) {
      const float alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] *= alpha;
    }
    const float ms = m == -INFINITY ? 0.f : m;
    float p[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = __builtin_amdgcn_exp2f(fmaf(sv[e], e < 8 ? ka : kc, -ms));
      if (decltype(masked)::value) p[e] = ok >> e & 1 ? p[e] : 0.f;  // (a scale of 0 times -inf)
      l += p[e];
    }
    uint4 ph[2], pl[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float y0 = p[8 * x + 2 * e], y1 = p[8 * x + 2 * e + 1];
        if (KVT == 2) {
          y0 *= x ? vc : va;
          y1 *= x ? vc : va;
        }
        split2(y0, y1, hi[e], lo[e]);
      }
      ph[x] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      pl[x] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
#pragma unroll
    for (int t = 0; t < NT; t += 2)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        // two groups of (2 dims 16 apart) x 4 slots: the two dims' operands
        const uint4 u = vt[x * TC + t * 64], v = vt[x * TC + t * 64 + 32];
        const uint4 o0 = make_uint4(u.x, u.y, v.x, v.y), o1 = make_uint4(u.z, u.w, v.z, v.w);
        acc[t] = mfma32(o0, ph[x], acc[t]);
        acc[t + 1] = mfma32(o1, ph[x], acc[t + 1]);
        acc[t] = mfma32(o0, pl[x], acc[t]);
        acc[t + 1] = mfma32(o1, pl[x], acc[t + 1]);
      }
    if (decltype(masked)::value && d0 >= 0 && bad_s) {
      // Infinities and NaN among the drafted values: 0 times them would reach the columns that do not
      // attend to them, so they are added column by column.
      for (int t = 0; t < 32 && d0 + t < n; ++t) {
        const int r = (t >> 3) * 4 + (t & 3), from = ((t >> 2) & 1) * 32 + cn;
        float pt = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (e == r) pt = p[e];
        pt = __shfl(pt, from, 64);
        const bool okt = (__shfl((int)ok, from, 64) >> r & 1) != 0;
#pragma unroll
        for (int y = 0; y < NT; ++y)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int d = 64 * (y >> 1) + 16 * (y & 1) + 32 * (e >> 3) + 8 * ((e >> 2) & 1) + 4 * h + (e & 3);
            const float v = widen(vd[(int64_t)(d0 + t) * a.vs + d]);
            if (okt && !(fabsf(v) < INFINITY)) acc[y][e] += pt * v;
          }
      }
    }
  };

  // this lane's tokens out of a pair's 32 bits
  auto own_bits = [&](uint32_t bits) {
    uint32_t ok = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) ok |= (bits >> (8 * (e >> 2) + 4 * h + (e & 3)) & 1u) << e;
    return ok;
  };
  const std::integral_constant<bool, false> full;
  const std::integral_constant<bool, true> masked;
  for (s0 = 0; s0 < ncache; s0 += SEG) {
    se = min(ncache, s0 + SEG);
    if (s0 > 0) __syncthreads();
    for (int i = tid; i < 2 * (se - s0); i += 64 * W) {
      const int id = min(max(a.page_table[(size_t)b * a.max_pages + p0 + min(2 * s0 + i, np - 1)], 0), a.num_pages - 1);
      id_s[i] = id;
      if (KVT == 2) {
        ksc_s[i] = a.ksc[(size_t)id * a.nkv + j];
        vsc_s[i] = a.vsc[(size_t)id * a.nkv + j];
      }
    }
    __syncthreads();
    Pair r0, r1;
    load_stage(s0, r0);
    load_stage(s0 + 1, r1);
    store_stage(s0, r0);
    load_stage(s0 + 2, r0);
    __syncthreads();
    auto step = [&](int s, Pair &r) {
      store_stage(s + 1, r);
      load_stage(s + 3, r);
      __builtin_amdgcn_sched_barrier(0);
      if (busy) compute(s, full, 0u, -1);
      __syncthreads();
    };
    const int end = min(se, nfull);
    int s = s0;
    for (; s + 1 < end; s += 2) {
      step(s, r1);
      step(s + 1, r0);
    }
    if (s < end) step(s, r1);
    if (end < se && busy)  // the candidate's last pair (in its buffer since the step before)
      compute(end, masked, own_bits((1u << (L - (p0 + 2 * end) * kPage)) - 1u), -1);
  }
  if (c == nc - 1) {
    for (int t0 = 0; t0 < n; t0 += 32) {
      __syncthreads();
      if (tid == 0) bad_s = 0;
      __syncthreads();
      store_draft(t0);
      __syncthreads();
      if (!busy) continue;
      uint32_t bits;
      const int own = tok - t0;
      if (a.mask) bits = a.mask[(tr.r0 + tok) * a.mask_words + (t0 >> 5)];
      else bits = own >= 31 ? ~0u : own < 0 ? 0u : (2u << own) - 1u;
      if (n - t0 < 32) bits &= (1u << (n - t0)) - 1u;
      compute(0, masked, own_bits(bits), t0);
    }
  }
  if (!present) return;
  {
    const uint32_t u = __float_as_uint(l);
    const auto t = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    l = __uint_as_float(t[0]) + __uint_as_float(t[1]);
  }
  const int64_t row = tr.r0 + tok, at = (row * a.nq + head) * a.slots + c;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 64 * (t >> 1) + 16 * (t & 1) + 32 * (i >> 1) + 8 * (i & 1) + 4 * h;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[t][4 * i + e] * (nc == 1 ? inv : 1.f);
      if (nc == 1) store4((T *)a.o + row * a.os + (int64_t)head * D + d, v);
      else store4(a.pacc + at * D + d, v);
    }
  if (nc > 1 && h == 0) a.pml[at] = make_float2(m, l);
}

// Joins the chunks of one (drafted token, q-head), one wave each: weights 2^(m - M) from one load
// per lane (at most 64 chunks), then the chunk sums in order.
template <int D, typename T>
__global__ __launch_bounds__(256) void k_tree_merge(TreeArgs a) {
  const int b = blockIdx.y, lane = threadIdx.x & 63;
  const int item = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (threadIdx.x >> 6));
  const TreeRows tr = tree_rows(a, b);
  const int t = item / a.nq, head = item - t * a.nq;
  const int npages = (tr.L + kPage - 1) / kPage;
  const int nc = tree_chunks(a, npages);
  if (t >= tr.n || nc == 1) return;
  const int64_t row = tr.r0 + t, at = (row * a.nq + head) * a.slots;
  const float2 ml = lane < nc ? a.pml[at + lane] : make_float2(-INFINITY, 0.f);
  const float M = wmax(ml.x);
  const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
  const float l = wsum(f * ml.y);
  constexpr int E = D / 64;
  float v[E] = {};
  const float *p = a.pacc + at * D + lane * E;
  for (int i = 0; i < nc; ++i) {
    const float w = lane_value(f, i);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] += w * p[(size_t)i * D + e];
  }
  T *o = (T *)a.o + row * a.os + (int64_t)head * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float y = l == 0.f ? 0.f : v[e] / l;
    if constexpr (sizeof(T) == 4) {
      o[e] = y;
    } else {
      uint32_t hi, lo;
      split2(y, 0.f, hi, lo);
      o[e] = (T)hi;
    }
  }
}

// ------------------------------------------------------------------------------- launch

struct TreePlan {
  int wide;    // waves of a k_tree_wide block, 0 = k_tree
  int nc;      // column tiles of a k_tree block
  int cols;    // columns of a block
  int blocks;  // column blocks of the longest draft
  int fill;    // blocks that fill the chip
  int unit;    // pages that a chunk is a multiple of
  int slots;   // chunk slots
};

// Kernel by the longest draft's columns. Chunk slots: what fills the chip eight times over if the
// batch's candidates were all as long as the table.
static TreePlan tree_plan(const Dims &dm, const kvprm_batch &b, const kvprm_tree &t) {
  TreePlan p;
  const int cols = t.max_rows * dm.g;
  p.wide = t.dtype == KVPRM_BF16 && dm.kvdt != 0 && cols > 32 ? (cols <= 64 ? 2 : 4) : 0;
  p.nc = cols <= 16 ? 1 : 2;
  p.cols = p.wide ? 32 * p.wide : 16 * p.nc;
  p.blocks = (cols + p.cols - 1) / p.cols;
  p.fill = p.wide ? 2048 / p.wide : 512;
  p.unit = p.wide ? 2 : 2 * kTreeWaves;
  const int64_t items = (int64_t)b.batch * dm.nkv * p.blocks;
  int64_t slots = (8 * p.fill + items - 1) / items;
  slots = min(slots, (int64_t)(b.max_pages + p.unit - 1) / p.unit);
  p.slots = (int)max((int64_t)1, min(slots, (int64_t)64));
  return p;
}

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

size_t tree_ws_bytes(const Dims &dm, const kvprm_batch &b, const kvprm_tree &t) {
  const TreePlan p = tree_plan(dm, b, t);
  if (p.slots == 1) return 256;
  const size_t parts = (size_t)t.num_rows * dm.nq * p.slots;
  return align256(parts * dm.d * 4) + align256(parts * 8);
}

static int cached_pages(const kvprm_batch &b, int i) {
  return b.lengths_host ? (b.lengths_host[i] + kPage - 1) / kPage : b.max_pages;
}

// Pages of a chunk: the fewest (multiples of p.unit) whose chunks leave the grid within p.fill blocks
// and each candidate within its slots.
static int tree_chunk_pages(const Dims &dm, const kvprm_batch &b, const TreePlan &p) {
  int longest = 0;
  for (int i = 0; i < b.batch; ++i) longest = max(longest, cached_pages(b, i));
  const int least = p.wide ? 16 : p.unit;
  int cp = max(least, ((longest + p.slots - 1) / p.slots + p.unit - 1) / p.unit * p.unit);
  const int64_t most = p.fill / ((int64_t)dm.nkv * p.blocks);
  for (;; cp += max(p.unit, cp / 8 / p.unit * p.unit)) {
    int64_t chunks = 0;
    for (int i = 0; i < b.batch; ++i) chunks += max(1, (cached_pages(b, i) + cp - 1) / cp);
    if (chunks <= max(most, (int64_t)b.batch) || cp >= longest) return cp;
  }
}

hipError_t launch_tree(const Dims &dm, const kvprm_kv_cache &c, const kvprm_batch &b, int layer,
                       const kvprm_tree &t, void *ws, hipStream_t s) {
  const TreePlan p = tree_plan(dm, b, t);
  const size_t tiles = (size_t)c.num_pages * dm.nkv;
  const size_t bytes = tiles * kPage * dm.d * (dm.kvdt == 0 ? 4 : dm.kvdt == 1 ? 2 : 1);
  TreeArgs a;
  a.kp = (const char *)c.k_pages + layer * bytes;
  a.vp = (const char *)c.v_pages + layer * bytes;
  a.ksc = dm.kvdt == 2 ? c.k_scale + layer * tiles : nullptr;
  a.vsc = dm.kvdt == 2 ? c.v_scale + layer * tiles : nullptr;
  a.B = b.batch;
  a.nkv = dm.nkv;
  a.g = dm.g;
  a.nq = dm.nq;
  a.num_pages = c.num_pages;
  a.page_table = b.page_table;
  a.max_pages = b.max_pages;
  a.lengths = b.lengths;
  a.q = t.q, a.k = t.k, a.v = t.v, a.o = t.o;
  a.qs = t.q_stride, a.ks = t.k_stride, a.vs = t.v_stride, a.os = t.o_stride;
  a.num_rows = t.num_rows;
  a.start = t.start;
  a.max_rows = t.max_rows;
  a.mask = t.mask;
  a.mask_words = t.mask_words;
  a.ginv = ((1u << 18) + dm.g - 1) / dm.g;
  a.chunk_pages = tree_chunk_pages(dm, b, p);
  a.slots = p.slots;
  a.pacc = (float *)ws;
  a.pml = (float2 *)((char *)ws + align256((size_t)t.num_rows * dm.nq * p.slots * dm.d * 4));
  int chunks = 1;
  int64_t items = 0;  // chunks of all candidates
  for (int i = 0; i < b.batch; ++i) {
    const int nc = max(1, (cached_pages(b, i) + a.chunk_pages - 1) / a.chunk_pages);
    chunks = max(chunks, nc);
    items += nc;
  }
  a.chunks = chunks;
  const dim3 grid((unsigned)(items * dm.nkv * p.blocks));
  const bool bf16 = t.dtype == KVPRM_BF16;
#define KVPRM_TREE(K_, D_, N_, T_) \
  hipLaunchKernelGGL((k_tree<K_, D_, N_, T_>), grid, dim3(64 * kTreeWaves), 0, s, a)
#define KVPRM_TREE_N(K_, D_, T_)                  \
  if (p.nc == 1) { KVPRM_TREE(K_, D_, 1, T_); }   \
  else { KVPRM_TREE(K_, D_, 2, T_); }
#define KVPRM_TREE_T(K_, D_)                      \
  if (bf16) { KVPRM_TREE_N(K_, D_, uint16_t) }    \
  else { KVPRM_TREE_N(K_, D_, float) }
#define KVPRM_TREE_D(K_)                          \
  if (dm.d == 64) { KVPRM_TREE_T(K_, 64) }        \
  else { KVPRM_TREE_T(K_, 128) }
#define KVPRM_WIDE(K_, D_)                                                                              \
  if (p.wide == 2) hipLaunchKernelGGL((k_tree_wide<K_, D_, 2>), grid, dim3(128), 0, s, a);              \
  else hipLaunchKernelGGL((k_tree_wide<K_, D_, 4>), grid, dim3(256), 0, s, a)
  if (p.wide) {
    if (dm.kvdt == 1 && dm.d == 64) { KVPRM_WIDE(1, 64); }
    else if (dm.kvdt == 1) { KVPRM_WIDE(1, 128); }
    else if (dm.d == 64) { KVPRM_WIDE(2, 64); }
    else { KVPRM_WIDE(2, 128); }
  } else if (dm.kvdt == 0) { KVPRM_TREE_D(0) }
  else if (dm.kvdt == 1) { KVPRM_TREE_D(1) }
  else { KVPRM_TREE_D(2) }
#undef KVPRM_WIDE
#undef KVPRM_TREE_D
#undef KVPRM_TREE_T
#undef KVPRM_TREE_N
#undef KVPRM_TREE
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || chunks == 1) return e;
  const dim3 mgrid((unsigned)(((int64_t)t.max_rows * dm.nq + 3) / 4), b.batch);
#define KVPRM_MERGE(D_)                                                                       \
  if (bf16) hipLaunchKernelGGL((k_tree_merge<D_, uint16_t>), mgrid, dim3(256), 0, s, a);      \
  else hipLaunchKernelGGL((k_tree_merge<D_, float>), mgrid, dim3(256), 0, s, a)
  if (dm.d == 64) { KVPRM_MERGE(64); }
  else { KVPRM_MERGE(128); }
#undef KVPRM_MERGE
  return hipGetLastError();
}

}  // namespace kvprm
