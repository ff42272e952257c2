// Attention of drafted tokens over the paged cache for gfx950: k_tree and k_tree_wide (chunks of cached pages
// and the drafted keys, by sequence, kv-head and columns; few columns and many) and k_tree_merge (the chunks'
// join).
#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

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
  int chunk_pages;         // most cached pages of a chunk (a multiple of unit)
  int block_cols;          // columns of a k_tree_wide block, a multiple of 32
  int unit;                // pages that chunks are multiples of: a step of every wave of the block
  int draft_tokens, draft_pages;  // so many drafted tokens (or a part) take a block as long as so many pages
  int chunks;              // chunks of the grid: a candidate has no more
  int slots;               // chunk slots of a (row, q-head) in the workspace (at least chunks)
  int part_rows;           // workspace rows of a candidate; 0: as the arrays' rows
  float *pacc;             // [row][q-head][slot][D] chunk sums
  float2 *pml;             // [row][q-head][slot] chunk maximum (log2 units) and sum
};

constexpr int kTreeWaves = 4;
constexpr int kTreeSegStages = 128;  // page pairs whose ids (and scales) a k_tree_wide block holds at a time
constexpr int kTreeSeg = 64 * kTreeWaves;  // pages whose ids a k_tree block's lanes hold at a time

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

// The workspace row of a candidate's first token.
__device__ __forceinline__ int part_row(const TreeArgs &a, int b, const TreeRows &r) {
  return a.part_rows ? b * a.part_rows : (int)r.r0;
}

// A candidate's cached pages in chunks of equal size (to a unit), as few as have at most chunk_pages
// each. The last chunk also takes the drafted tokens and has as many pages fewer as these take time, none
// if need be; a cache of one chunk keeps them in it.
struct TreeSplit {
  int chunks, pages;  // pages of each chunk but the last
};
__host__ __device__ inline int draft_chunks(int npages, int extra, int pages) {  // chunks of at most `pages`
  const int cached = (npages + pages - 1) / pages;
  return cached <= 1 ? 1 : min(cached + 1, (npages + extra + pages - 1) / pages);
}
__device__ __forceinline__ TreeSplit tree_split(const TreeArgs &a, const TreeRows &r) {
  const int npages = (r.L + kPage - 1) / kPage;
  const int extra = (r.n + a.draft_tokens - 1) / a.draft_tokens * a.draft_pages;
  const int most = min(a.chunks, draft_chunks(npages, extra, a.chunk_pages));
  TreeSplit s = {1, npages};
  if (most > 1) {
    s.pages = (npages + extra + most * a.unit - 1) / (most * a.unit) * a.unit;
    s.chunks = draft_chunks(npages, extra, s.pages);
  }
  return s;
}

// The block's work: candidate, kv-head, chunk of its cached pages and block of its columns. The grid is
// one-dimensional and holds the blocks that exist, candidate by candidate (a scan over the lanes finds the
// candidate), then blocks without work, which leave at once: a grid of (chunk, column block, candidate) sides
// leaves them in a pattern that keeps part of the compute units idle on ragged batches. Blocks go to the
// eight XCDs in turn; the column blocks of one chunk, which read the same pages, lie eight apart, so
// that they share an L2.
struct TreeItem {
  int b, j, chunk, colblock;
  TreeRows rows;
};
__device__ __forceinline__ bool tree_item(const TreeArgs &a, int cols_per_block, TreeItem &it) {
  const int lane = threadIdx.x & 63;
  int id = blockIdx.x;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    int items_l = 0, cb_l = 0;
    TreeRows r = {0, 0, 0};
    if (b0 + lane < a.B) {
      r = tree_rows(a, b0 + lane);
      if (r.n > 0) {
        items_l = tree_split(a, r).chunks * a.nkv;
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
    it.rows.L = lane_value(r.L, k);
    it.rows.n = lane_value(r.n, k);
    it.rows.r0 = lane_value((int)r.r0, k);
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

// Infinities among cached bf16 values. A weight is a sum of bf16 terms, of which the lower ones may be 0 or negative,
// so that its product with an infinity can be NaN where the definition has the infinity. Sums that ended as NaN
// therefore look up which infinities their dim holds: a wave reads the value tiles of its pages once more, at the
// memory's rate but for the tiles that hold something not finite. (Where all sums are finite this costs their test.)
template <int N>
struct Special {
  uint64_t plus = 0, minus = 0, nan = 0;  // bit y: the dim of this lane's y-th sum
  // The first `slots` slots of a bf16 value tile (see kvprm_kv_cache); dim(y): dim of the y-th sum.
  template <int D, typename F>
  __device__ __forceinline__ void look(const uint16_t *tile, int slots, int lane, F dim) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const uint4 x = ((const uint4 *)tile)[i * 64 + lane];
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) any = any || (w[e] & 0x7F80u) == 0x7F80u || (w[e] & 0x7F800000u) == 0x7F800000u;
    }
    if (!__any(any)) return;
#pragma unroll 1
    for (int y = 0; y < N; ++y) {
      const int m = dim(y);
#pragma unroll 1
      for (int s = 0; s < slots; ++s) {
        const uint32_t v = tile[((((m >> 5) * 4 + (s >> 2)) * 16 + (m & 15)) * 2 + (m >> 4 & 1)) * 4 + (s & 3)];
        if ((v & 0x7F80u) != 0x7F80u) continue;
        const uint64_t bit = (uint64_t)1 << y;
        if (v & 0x7Fu) nan |= bit;
        else if (v >> 15) minus |= bit;
        else plus |= bit;
      }
    }
  }
  __device__ __forceinline__ float mend(float sum, int y) const {  // the y-th sum
    const bool p = plus >> y & 1, q = minus >> y & 1;
    return sum == sum || (nan >> y & 1) || p == q ? sum : p ? INFINITY : -INFINITY;
  }
};

// o = softmax(q K^T / sqrt(d)) V for NC tiles of 16 columns (drafted token, q-head of the kv-head's
// group), over one chunk of a candidate's cached pages; the last chunk also takes the drafted keys.
// A block's four waves take page pairs in turn and join their softmax states in LDS, so that a chunk is
// one partial result.
// A page pair (32 tokens) is one step: S = K Q^T, a running softmax in registers, O^T += V^T P^T, all
// on the matrix cores with the cache's tiles as they lie in memory (see kvprm_attn.hip), the next pair's loads
// in flight. Bound by memory on long caches: 8 of 16384 to 32768 tokens, 4 kv-heads of 128 dims, bf16, 28
// columns (410 MB): 90 us, 4.5 TB/s. On short ones by the chain of loads, products and join: 1103 tokens,
// 16 drafted, 8 kv-heads, 32 columns in two blocks of 16: 8 us, and 4 for k_tree_merge.
template <int KVT, int D, int NC, typename T>
__global__ __launch_bounds__(64 * kTreeWaves, KVT == 3 ? 2 : 1) void k_tree(TreeArgs a) {
  constexpr int NKB = D / 32, NDB = D / 16, W = kTreeWaves;
  constexpr int QT = Terms<T>::Q, PT = Terms<T>::P;
  constexpr size_t TILE = tile_bytes(KVT, D);
  __shared__ floatx4 sacc[W][NC][NDB][64];
  __shared__ float2 sml[W][NC * 16];
  TreeItem it;
  if (!tree_item(a, 16 * NC, it)) return;
  const int b = it.b, j = it.j, c = it.chunk;
  const TreeRows tr = it.rows;
  const int L = tr.L, n = tr.n, g = a.g;
  const int cols = n * g, col0 = it.colblock * 16 * NC;
  const int npages = (L + kPage - 1) / kPage;
  const TreeSplit sp = tree_split(a, tr);
  const int nc = sp.chunks;
  const int p0 = c * sp.pages, np = max(0, min(sp.pages, npages - p0));
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
    const int first = p0 + seg, sn = min(kTreeSeg, np - seg);  // pages of this segment
    if constexpr (KVT == 0) {
      // wave w takes pages w, w + W, ...; lane i holds the id of its i-th page
      const int mine = (sn - w + W - 1) / W;
      if (mine <= 0) continue;
      const int id_l =
          min(max(a.page_table[(size_t)b * a.max_pages + first + min(w + W * lane, sn - 1)], 0), a.num_pages - 1);
      float qf[NC][D / 4];
#pragma unroll
      for (int ct = 0; ct < NC; ++ct) query32<D>(qrow(ct), cq, present[ct], qf[ct]);
      for (int i = 0; i < mine; ++i) {
        const size_t tile = ((size_t)lane_value(id_l, i) * a.nkv + j) * TILE;
        const float4 *kt = (const float4 *)(a.kp + tile), *vt = (const float4 *)(a.vp + tile);
        const int t0 = (first + w + W * i) * kPage + 4 * cq;
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
      const int id_l = min(max(a.page_table[(size_t)b * a.max_pages + first + pg], 0), a.num_pages - 1);
      float ksc_l = 0.f, vsc_l = 0.f;
      if (KVT == 2) {
        ksc_l = a.ksc[(size_t)id_l * a.nkv + j];
        vsc_l = a.vsc[(size_t)id_l * a.nkv + j];
      }
      auto load_pair = [&](int i, PairOf<KVT, D> &r) {
        const int ia = 2 * min(i, mine - 1);
        const size_t ta = ((size_t)lane_value(id_l, ia) * a.nkv + j) * TILE;
        const size_t tb = ((size_t)lane_value(id_l, ia + 1) * a.nkv + j) * TILE;
        load_pair_of<KVT, D, false>(a.kp + ta, a.kp + tb, a.vp + ta, a.vp + tb, lane, r);
      };
      PairOf<KVT, D> r0, r1;
      load_pair(0, r0);
      uint4 qo[NC][QT][NKB];
#pragma unroll
      for (int ct = 0; ct < NC; ++ct) {
        const T *qr = qrow(ct);
#pragma unroll
        for (int kk = 0; kk < NKB; ++kk) {
          const int dim = key_dim<KVT, D>(kk, cq);
          if constexpr (QT == 1) {
            const uint4 v = *(const uint4 *)(qr + dim);
            qo[ct][0][kk] = present[ct] ? v : make_uint4(0, 0, 0, 0);
          } else {
            float v[8];
            load4((const float *)qr + dim, v);
            load4((const float *)qr + dim + 4, v + 4);
            if (KVT == 3)  // (see kScoreShift4)
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] *= 1.f / kScoreUnit4;
            uint32_t t[3][4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              split3(present[ct] ? v[2 * e] : 0.f, present[ct] ? v[2 * e + 1] : 0.f, t[0][e], t[1][e], t[2][e]);
#pragma unroll
            for (int x = 0; x < QT; ++x) qo[ct][x][kk] = make_uint4(t[x][0], t[x][1], t[x][2], t[x][3]);
          }
        }
      }
      // 4-bit pairs: keys and values become operands 32 dims at a time (all at once they would take the registers of
      // two waves a unit), and only the candidate's last pair masks slots. In blocks of 32 columns, which they had
      // then: 8 caches of 16384 to 32768 tokens, 4 drafted, 28 columns, 59 us a call in the other types' order, 53
      // so.
      auto compute4 = [&](int i, const PairOf<KVT, D> &r, auto masked) {
        constexpr bool TAIL = decltype(masked)::value;
        if constexpr (KVT == 3) {
          const int left = L - (first + 2 * (w + W * i)) * kPage - 4 * cq;  // (as below)
          const float rs4 = QT == 1 ? rs : rs * kScoreUnit4;
          floatx4 sa[NC], sb[NC];
#pragma unroll
          for (int ct = 0; ct < NC; ++ct) sa[ct] = sb[ct] = floatx4{0.f, 0.f, 0.f, 0.f};
          const float ka = scale_of<0>(r.ks[0]), kb = scale_of<0>(r.ks[1]);
#pragma unroll
          for (int kk = 0; kk < NKB; ++kk) {
            const uint4 a4 = keys4(word(r.k[0], kk), ka), b4 = keys4(word(r.k[1], kk), kb);
#pragma unroll
            for (int x = 0; x < QT; ++x)
#pragma unroll
              for (int ct = 0; ct < NC; ++ct) {
                sa[ct] = mfma16(a4, qo[ct][x][kk], sa[ct]);
                sb[ct] = mfma16(b4, qo[ct][x][kk], sb[ct]);
              }
          }
          uint4 P[NC][PT];
#pragma unroll
          for (int ct = 0; ct < NC; ++ct) {
            float p[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              p[e] = sa[ct][e] * rs4;
              p[4 + e] = sb[ct][e] * rs4;
              if (TAIL) {
                p[e] = left > e ? p[e] : -INFINITY;
                p[4 + e] = left > 16 + e ? p[4 + e] : -INFINITY;
              }
            }
            st[ct].template weights<8>(p);
            uint32_t t[3][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if constexpr (PT == 2) split2(p[2 * e], p[2 * e + 1], t[0][e], t[1][e]);
              else split3(p[2 * e], p[2 * e + 1], t[0][e], t[1][e], t[2][e]);
            }
#pragma unroll
            for (int x = 0; x < PT; ++x) P[ct][x] = make_uint4(t[x][0], t[x][1], t[x][2], t[x][3]);
          }
          const uint32_t a0 = (left > 0 ? 0xFFFFu : 0u) | (left > 1 ? 0xFFFF0000u : 0u);
          const uint32_t a1 = (left > 2 ? 0xFFFFu : 0u) | (left > 3 ? 0xFFFF0000u : 0u);
          const uint32_t b0 = (left > 16 ? 0xFFFFu : 0u) | (left > 17 ? 0xFFFF0000u : 0u);
          const uint32_t b1 = (left > 18 ? 0xFFFFu : 0u) | (left > 19 ? 0xFFFF0000u : 0u);
#pragma unroll
          for (int g4 = 0; g4 < NKB; ++g4) {
            uint2 A[2], B[2];
            values4(word(r.v[0], g4), word(r.vs[0], g4), A[0], A[1]);
            values4(word(r.v[1], g4), word(r.vs[1], g4), B[0], B[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint4 v = make_uint4(A[h].x, A[h].y, B[h].x, B[h].y);
              if (TAIL) v = make_uint4(v.x & a0, v.y & a1, v.z & b0, v.w & b1);
#pragma unroll
              for (int x = 0; x < PT; ++x)
#pragma unroll
                for (int ct = 0; ct < NC; ++ct)
                  st[ct].acc[2 * g4 + h] = mfma16(v, P[ct][x], st[ct].acc[2 * g4 + h]);
            }
          }
        }
      };
      auto compute = [&](int i, const PairOf<KVT, D> &r) {
        if constexpr (KVT == 3) {
          if ((first + 2 * (w + W * i) + 2) * kPage > L) compute4(i, r, std::integral_constant<bool, true>{});
          else compute4(i, r, std::integral_constant<bool, false>{});
          return;
        }
        uint4 KA[NKB], KB[NKB];
        uint2 VA[NDB], VB[NDB];
        unpack_pair_of<KVT, D>(r, KA, KB, VA, VB);
        const int la = 2 * i;
        const float sca = KVT == 2 ? lane_value(ksc_l, la) * rs : rs;
        const float scb = KVT == 2 ? lane_value(ksc_l, la + 1) * rs : rs;
        const int t0 = (first + 2 * (w + W * i)) * kPage;
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

  if constexpr (KVT == 1) {
    float z[4] = {0.f, 0.f, 0.f, 0.f};  // NaN where a sum is not finite
#pragma unroll
    for (int ct = 0; ct < NC; ++ct)
#pragma unroll
      for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = fmaf(st[ct].acc[nb][e], 0.f, z[e]);
    if (__any((z[0] + z[1]) + (z[2] + z[3]) != 0.f)) {
      Special<NDB * 4> sp;
      for (int i = 0; i < np; ++i) {
        if ((i >> 1) % W != w) continue;  // (a segment is a multiple of W pairs)
        const int id = min(max(a.page_table[(size_t)b * a.max_pages + p0 + i], 0), a.num_pages - 1);
        sp.template look<D>((const uint16_t *)(a.vp + ((size_t)id * a.nkv + j) * TILE), min(kPage, L - (p0 + i) * kPage),
                            lane, [&](int y) { return 16 * (y >> 2) + 4 * cq + (y & 3); });
      }
#pragma unroll
      for (int ct = 0; ct < NC; ++ct)
#pragma unroll
        for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) st[ct].acc[nb][e] = sp.mend(st[ct].acc[nb][e], 4 * nb + e);
    }
  }

  // the drafted keys, 16 at a time, in fp32 (T^2 products beside T L: the fp32 matrix instructions
  // need no split); wave w takes column tile w % NC and every W / NC-th tile of keys
  if (c == nc - 1) {
    const T *kd = (const T *)a.k + tr.r0 * a.ks + (int64_t)j * D;
    const T *vd = (const T *)a.v + tr.r0 * a.vs + (int64_t)j * D;
    for (int t0 = 16 * (w / NC); t0 < n; t0 += 16 * (W / NC)) {
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
        if (ct != w % NC) continue;
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
    const int64_t at = ((int64_t)(part_row(a, b, tr) + tok[ct]) * a.nq + head[ct]) * a.slots + c;
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
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ floatx16 mfma32(const uint4 &a, const uint4 &b, const floatx16 &c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 mfma32h(const uint4 &a, const uint4 &b, const floatx16 &c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a),
                                                __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t half2(float x, float y) {  // nearest even
  typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
  typedef float f32x2v __attribute__((ext_vector_type(2)));
  const f32x2v v = {x, y};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, halfx2));
}
template <bool HIGH>
__device__ __forceinline__ uint32_t fp8x2_to_half2(uint32_t word) {  // (every e4m3 value is an fp16 value)
  typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
  const halfx2 v = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, 1.0f, HIGH);
  return __builtin_bit_cast(uint32_t, v);
}

// The same for drafts of many columns (bf16 rows): here the waves share the pages and split the
// columns, 32 each. A stage is a page pair (32 tokens) in LDS as 16-bit tiles in the stored order, double
// buffered, the next pairs' loads in flight while one is computed. 32x32x16 products: S = K Q^T (a lane holds
// tokens 8 i + 4 h + e, h = lane / 32, of column lane % 32), softmax, O^T += V^T P^T, tokens in S's order
// (8 slots 4 h.., 8 + 4 h.. of one page are one operand). bf16 caches: P in two bf16 terms (16 bits; one
// term would add an error the size of the result's own rounding). fp8 caches: keys widened to bf16, values to
// fp16, exactly, and P in fp16 (11 bits), half the products: 8 caches of 16384 to 32768 tokens, 4 kv-heads of
// 128 dims, 64 drafted tokens of 7 query heads each: 273 us, 675 TFLOP/s; from bf16 caches 330 us, 560 TFLOP/s (fp16
// values from those too, with an exponent per tile: 357 and more). Drafted values stay bf16 over fp8 caches too (two-
// term weights): as fp16 they would need an exponent that all of them share, and the largest of them would push others
// out of fp16's range, those also that a token sees without seeing the largest.
// Bound by vector instructions (about 115 a stage and wave at D = 128, bf16, 160 at D = 64, fp8, beside 24 and 8
// products) and by how far the two or three waves of a SIMD overlap them with products: a ring of four stages
// with half the barriers, wave priorities and waves in two groups taking turns all measured the same.
// The drafted keys are stages of their own behind the last chunk's pages, laid out as a page pair.
template <int KVT, int D, int W>
__global__ __launch_bounds__(64 * W, D == 64 ? 3 : 2) void k_tree_wide(TreeArgs a) {
  typedef uint16_t T;
  constexpr int KS = D / 16, NT = D / 32, TC = 2 * D;  // k steps, output tiles, 16-byte groups of a bf16 tile
  constexpr int SC = KVT == 1 ? 2 * TC : KVT == 2 ? TC : TC / 2;  // 16-byte groups of a pair in memory (codes)
  // of these per thread, K or V (4-bit: a lane's codes and scales)
  constexpr int NLC = KVT == 3 ? 2 : (SC + 64 * W - 1) / (64 * W);
  constexpr int SEG = kTreeSegStages;
  constexpr bool HALF = KVT == 2;  // values and weights in fp16
  // Pairs that half of the waves can move: the first half of them moves keys, the others values.
  constexpr bool ROLES = KVT != 3 && 2 * SC <= 64 * W;
  // 4-bit pairs: a wave widens words of 8 codes of one page, W4 of the keys and W4 of the values for each lane. (With
  // whole pages to a wave, two waves for keys and two for values, all waited at each stage's barrier for those with
  // the values, which take more instructions: 8 caches of 16384 to 32768 tokens as below 309 us instead of 282.)
  constexpr int W4 = D / 64;
  static_assert(KVT != 3 || W == 4, "4-bit stages: two waves a page");
  __shared__ uint4 kb[2][2 * TC], vb[2][2 * TC];
  __shared__ int id_s[2 * SEG + 12];                    // page ids of a segment
  __shared__ float ksc_s[KVT == 2 ? 2 * SEG + 12 : 1];  // key scales / sqrt(d), log2 units
  __shared__ float vsc_s[KVT == 2 ? 2 * SEG + 12 : 1];  // value scales: factor and exponent
  __shared__ int vex_s[KVT == 2 ? 2 * SEG + 12 : 1];
  // Largest unit so far. Others stay within 2^-kUnits of it: acc, which holds up to 2^40 (2^18 tokens' weights below
  // 2^13 times codes), moves to each, and would overflow in one further below. (What a unit kept higher loses is below
  // 2^-(kUnits + 20) of the largest values; at 24 that was all of a page of small values whose tokens had the weight.)
  constexpr int kUnits = 80, kNoUnit = -1000;
  __shared__ int base_s;
  __shared__ int bad_s;
  TreeItem it;
  if (!tree_item(a, a.block_cols, it)) return;
  const int b = it.b, j = it.j, c = it.chunk;
  const TreeRows tr = it.rows;
  const int L = tr.L, n = tr.n, g = a.g;
  const int npages = (L + kPage - 1) / kPage;
  const TreeSplit sp = tree_split(a, tr);
  const int nc = sp.chunks;
  const int p0 = c * sp.pages, np = max(0, min(sp.pages, npages - p0));
  const int tid = threadIdx.x, lane = tid & 63, cn = lane & 31, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cols = n * g, col0 = it.colblock * a.block_cols + w * 32;
  const bool busy = col0 < cols && w * 32 < a.block_cols;
  struct Column {  // a lane's column: drafted token and q-head
    bool present;
    int tok, head;
  };
  auto column = [&](int lane) {
    const int col = col0 + (lane & 31);
    Column r = {busy && col < cols, 0, j * g};
    if (r.present) {
      r.tok = (int)(((uint32_t)col * a.ginv) >> 18);
      r.head += col - r.tok * g;
    }
    return r;
  };
  const float rs = kLog2e / sqrtf((float)D);
  const int ncache = (np + 1) >> 1;                    // stages of cached pages
  const int nfull = max(0, L - p0 * kPage) >> 5;       // of these, the first without a slot at or past L
  const T *kd = (const T *)a.k + tr.r0 * a.ks + (int64_t)j * D;
  const T *vd = (const T *)a.v + tr.r0 * a.vs + (int64_t)j * D;

  uint4 qo[KS];
  {
    const Column my = column(lane);
    const T *q = (const T *)a.q + (tr.r0 + my.tok) * a.qs + (int64_t)my.head * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const uint4 v = *(const uint4 *)(q + 16 * ks + 8 * h);
      qo[ks] = my.present ? v : make_uint4(0, 0, 0, 0);
    }
  }
  // A stage's keys or values in registers, as 16-byte groups in memory order. (No branch around loads,
  // which would join registers still in flight: stages past the segment's end repeat its last page.)
  struct Half {
    uint4 g[NLC];
  };
  int s0 = 0, se = 0;         // the segment's stages
  int kid_l = 0, vid_l = 0;   // lane i: page id i of the 64 that the key (value) loads are in
  auto load_words = [](const char *p) {  // W4 of them
    if constexpr (W4 == 1) return make_uint4(*(const uint32_t *)p, 0, 0, 0);
    else return load_bytes<4 * W4, false>(p);
  };
  auto load_half = [&](auto VAL, const char *pool, int s, int &id_l, Half &r) {
    const int i = 2 * (s - s0);
    if ((i & 63) == 0) id_l = id_s[min(i + lane, 2 * SEG + 11)];
    constexpr size_t TILE = tile_bytes(KVT, D);
    if constexpr (KVT == 3) {
      const char *t = pool + ((size_t)lane_value(id_l, (i & 63) + (w & 1)) * a.nkv + j) * TILE;
      const int at = (w >> 1) * 4 * W4;
      if (decltype(VAL)::value) {
        r.g[0] = load_words(t + at + value_code4<D>(lane));
        r.g[1] = load_words(t + at + value_scale4<D>(lane));
      } else {
        r.g[0] = load_words(t + at + key_code4<D>(lane));
        r.g[1].x = *(const uint8_t *)(t + key_scale4<D>(lane));
      }
      return;
    }
    const int ia = lane_value(id_l, i & 63), ib = lane_value(id_l, (i & 63) + 1);
#pragma unroll
    for (int k = 0; k < NLC; ++k) {
      // this wave's first group
      const int i0 = (k * 64 * W + w * 64) % SC;
      const char *t = pool + ((size_t)(i0 >= SC / 2 ? ib : ia) * a.nkv + j) * TILE + (i0 % (SC / 2)) * 16;
      r.g[k] = *(const uint4 *)(t + (uint32_t)(lane * 16));
    }
  };
  auto load_keys = [&](int s, Half &r) { load_half(std::false_type(), a.kp, s, kid_l, r); };
  auto load_values = [&](int s, Half &r) { load_half(std::true_type(), a.vp, s, vid_l, r); };
  // Keys: group (8 dims c, page, slot) at 32 c + 16 page + slot: step ks of the products reads groups
  // 64 ks + lane.
  auto store_keys = [&](int s, const Half &r) {
    uint4 *kt = kb[s & 1];
    if constexpr (KVT == 3) {
      const float sc = scale_of<0>(r.g[1].x);
#pragma unroll
      for (int x = 0; x < W4; ++x)
        kt[((lane >> 4) * (D / 32) + (w >> 1) * W4 + x) * 32 + (w & 1) * 16 + (lane & 15)] = keys4(word(r.g[0], x), sc);
      return;
    }
#pragma unroll
    for (int k = 0; k < NLC; ++k) {
      const int i0 = (k * 64 * W + w * 64) % SC, i = i0 % (SC / 2) + lane;
      const int at = (i >> 4) * (KVT == 1 ? 32 : 64) + (i0 >= SC / 2 ? 16 : 0) + (i & 15);
      const uint4 x = r.g[k];
      if (KVT == 1) {
        kt[at] = x;
      } else {  // 16 dims of a slot -> two groups of 8
        kt[at] = make_uint4(fp8x2_to_bf16x2<false>(x.x), fp8x2_to_bf16x2<true>(x.x),
                            fp8x2_to_bf16x2<false>(x.y), fp8x2_to_bf16x2<true>(x.y));
        kt[at + 32] = make_uint4(fp8x2_to_bf16x2<false>(x.z), fp8x2_to_bf16x2<true>(x.z),
                                 fp8x2_to_bf16x2<false>(x.w), fp8x2_to_bf16x2<true>(x.w));
      }
    }
  };
  // Values: 4 slots 4 q .. of dim 32 t + mm of a page, 8 bytes, at [page][t][q & 1][mm][q >> 1]: the
  // product of page and tile t reads groups 64 t + lane of the page.
  auto value_at = [&](int t, int mm, int q) { return ((t * 2 + (q & 1)) * 32 + mm) * 2 + (q >> 1); };
  auto store_values = [&](int s, const Half &r) {
    if constexpr (KVT == 3) {
      uint2 *vt = (uint2 *)(vb[s & 1] + ((w & 1) ? TC : 0));
      const int q = lane >> 4, mm = lane & 15;
      // slots at or past L may hold anything: they become zeros
      const int have = s >= nfull ? L - (p0 + 2 * s + (w & 1)) * kPage - 4 * q : kPage;
      const uint32_t m0 = (have > 0 ? 0xFFFFu : 0u) | (have > 1 ? 0xFFFF0000u : 0u);
      const uint32_t m1 = (have > 2 ? 0xFFFFu : 0u) | (have > 3 ? 0xFFFF0000u : 0u);
#pragma unroll
      for (int x = 0; x < W4; ++x) {  // dims mm and mm + 16 of tile t
        const int t = (w >> 1) * W4 + x;
        uint2 lo, hi;
        values4(word(r.g[0], x), word(r.g[1], x), lo, hi);
        vt[value_at(t, mm, q)] = make_uint2(lo.x & m0, lo.y & m1);
        vt[value_at(t, mm + 16, q)] = make_uint2(hi.x & m0, hi.y & m1);
      }
      return;
    }
#pragma unroll
    for (int k = 0; k < NLC; ++k) {
      const int i0 = (k * 64 * W + w * 64) % SC, i = i0 % (SC / 2) + lane;
      const bool second = i0 >= SC / 2;
      uint2 *vt = (uint2 *)(vb[s & 1] + (second ? TC : 0));
      const int q = (i >> 4) & 3, mm = i & 15;
      uint4 x = r.g[k];
      if (s >= nfull) {  // slots at or past L may hold anything: they become zeros
        const int have = L - (p0 + 2 * s + second) * kPage - 4 * q;
        if (KVT == 1) {
          const uint32_t m0 = (have > 0 ? 0xFFFFu : 0u) | (have > 1 ? 0xFFFF0000u : 0u);
          const uint32_t m1 = (have > 2 ? 0xFFFFu : 0u) | (have > 3 ? 0xFFFF0000u : 0u);
          x = make_uint4(x.x & m0, x.y & m1, x.z & m0, x.w & m1);
        } else {
          const uint32_t m0 = have <= 0 ? 0u : have > 3 ? ~0u : (1u << 8 * have) - 1u;
          x = make_uint4(x.x & m0, x.y & m0, x.z & m0, x.w & m0);
        }
      }
      if (KVT == 1) {  // dims mm and mm + 16 of tile t
        const int t = i0 % (SC / 2) >> 6;
        vt[value_at(t, mm, q)] = make_uint2(x.x, x.y);
        vt[value_at(t, mm + 16, q)] = make_uint2(x.z, x.w);
      } else {  // dims mm, mm + 16, .. + 48 of 64
        const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          vt[value_at(2 * (i >> 6) + (e >> 1), mm + 16 * (e & 1), q)] =
              make_uint2(fp8x2_to_half2<false>(y[e]), fp8x2_to_half2<true>(y[e]));
      }
    }
  };
  const int role = ROLES ? w / (W / 2) : 0;
  auto load_own = [&](int s, Half &r) { load_half(std::false_type(), role ? a.vp : a.kp, s, kid_l, r); };
  auto store_own = [&](int s, const Half &r) {
    if (role) store_values(s, r);
    else store_keys(s, r);
  };
  // 32 drafted tokens from t0 on as a page pair in buffer 0, all in bf16.
  auto store_draft = [&](int t0) {
    constexpr int ND = (2 * TC + 64 * W - 1) / (64 * W);
    uint4 *kt = kb[0];
    uint16_t *vt = (uint16_t *)vb[0];
    uint4 rv[ND];
    bool bad = false;
#pragma unroll
    for (int k = 0; k < ND; ++k) {
      const int i = k * 64 * W + tid, t = i / (D / 8), e = 8 * (i % (D / 8));
      rv[k] = make_uint4(0, 0, 0, 0);
      uint4 rk = rv[k];
      if (i < 2 * TC && t0 + t < n) {
        rk = *(const uint4 *)(kd + (t0 + t) * a.ks + e);
        rv[k] = *(const uint4 *)(vd + (t0 + t) * a.vs + e);
      }
      if (i < 2 * TC) kt[(e >> 3) * 32 + t] = rk;
      uint32_t *x = (uint32_t *)&rv[k];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        // infinities and NaN leave the product (see below)
        if ((x[y] & 0x7F80u) == 0x7F80u) bad = true, x[y] &= 0xFFFF0000u;
        if ((x[y] & 0x7F800000u) == 0x7F800000u) bad = true, x[y] &= 0xFFFFu;
      }
    }
    if (bad) bad_s = 1;
#pragma unroll
    for (int k = 0; k < ND; ++k) {
      const int i = k * 64 * W + tid, t = i / (D / 8), e = 8 * (i % (D / 8)), sl = t & 15;
      if (i >= 2 * TC) continue;
      const uint32_t *x = (const uint32_t *)&rv[k];
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const int mm = e + y;
        vt[((t >> 4) * 2 * TC + value_at(mm >> 5, mm & 31, sl >> 2)) * 4 + (sl & 3)] =
            (uint16_t)(x[y >> 1] >> (16 * (y & 1)));
      }
    }
  };

  float m = -INFINITY, l = 0.f;
  floatx16 acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
  // fp16 values: acc is in units of 2^unit, the exponent that values or their scales were divided by.
  int unit = 0;
  auto to_unit = [&](int to) {
    if (!HALF || to == unit) return;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[t][e] = ldexpf(acc[t][e], unit - to);  // (exact)
    unit = to;
  };

  // The pair in buffer `buf`: its keys as operands, and from them the scores, unscaled.
  auto keys = [&](int buf, uint4 (&ko)[KS]) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) ko[ks] = kb[buf][ks * 64 + lane];
  };
  auto scores = [&](const uint4 (&ko)[KS], floatx16 &sv) {
#pragma unroll
    for (int e = 0; e < 16; ++e) sv[e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) sv = mfma32(ko[ks], qo[ks], sv);
  };
  // The largest of a column's scores sv, of pages with scales ka, kc (positive; -inf stays -inf).
  auto largest = [&](const floatx16 &sv, float ka, float kc) {
    float ma = sv[0], mb = sv[8];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
      ma = fmaxf(ma, sv[e]);
      mb = fmaxf(mb, sv[8 + e]);
    }
    const float mx = fmaxf(ma * ka, mb * kc);
    const uint32_t u = __float_as_uint(mx);
    const auto t = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
  };
  // The weights are 2^(score - m), and m moves only once a score lies more than a limit above it, which leaves out
  // most of the rescaling. bf16 weights: m lies 12 above the largest score when it is set and moves when one passes
  // it; the weights stay below 1, so that values near fp32's largest stay finite. fp16 weights (H): m lies 8 below
  // and moves when a score comes to lie more than 12 above it; the weights stay below 2^12, and those that fp16
  // holds with fewer bits, below 2^-14, are 2^-22 of the largest or less.
  auto new_max = [&](auto H, float mx) {
    if (__any(mx > (decltype(H)::value ? m + 12.f : m))) {
      const float mn = fmaxf(m, decltype(H)::value ? mx - 8.f : mx + 12.f);
      const float alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] *= alpha;
    }
  };
  // P's operands by page: fp16 values (H) take the weights in fp16 (times their pages' scales va, vc), bf16
  // values in two bf16 terms.
  typedef std::integral_constant<bool, HALF> Cached;
  typedef std::integral_constant<bool, false> Drafted;
  auto operands = [&](auto H, const float (&p)[16], float va, float vc, uint4 (&ph)[2], uint4 (&pl)[2]) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y0 = p[8 * x + 2 * e], y1 = p[8 * x + 2 * e + 1];
        if constexpr (decltype(H)::value) {
          const float f = x ? vc : va;
          hi[e] = half2(y0 * f, y1 * f);
          lo[e] = 0;
        } else {
          split2(y0, y1, hi[e], lo[e]);
        }
      }
      ph[x] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      pl[x] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
  };
  auto values = [&](int buf, uint4 (&vo)[2][NT]) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int t = 0; t < NT; ++t) vo[x][t] = vb[buf][x * TC + t * 64 + lane];
  };
  // (ua, uc: the units that the two pages' products come in)
  auto products = [&](auto H, const uint4 (&vo)[2][NT], const uint4 (&ph)[2], const uint4 (&pl)[2], int ua, int uc) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      to_unit(x ? uc : ua);
#pragma unroll
      for (int t = 0; t < NT; ++t)
        acc[t] = decltype(H)::value ? mfma32h(vo[x][t], ph[x], acc[t]) : mfma32(vo[x][t], ph[x], acc[t]);
      if (!decltype(H)::value)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = mfma32(vo[x][t], pl[x], acc[t]);
    }
  };
  // Scales of stage s's keys and values (s < 0: drafted tokens).
  struct Scales {
    float ka, kc, va, vc;
    int ua, uc;
  };
  auto scales = [&](int s) {
    Scales r = {rs, rs, 1.f, 1.f, 0, 0};
    if (KVT == 2 && s >= 0) {
      const int i = 2 * (s - s0);
      r.ka = ksc_s[i], r.kc = ksc_s[i + 1];
      r.va = vsc_s[i], r.vc = vsc_s[i + 1];
      r.ua = __builtin_amdgcn_readfirstlane(vex_s[i]), r.uc = __builtin_amdgcn_readfirstlane(vex_s[i + 1]);
    }
    return r;
  };
  // A pair of which only the tokens of `ok` (bit r: this lane's r-th) count: the candidate's last cached
  // one (stage s), or (s < 0) the drafted tokens from d0 on.
  auto compute_masked = [&](auto H, int s, int buf, uint32_t ok, int d0) {
    floatx16 sv;
    uint4 ko[KS], vo[2][NT];
    keys(buf & 1, ko);
    scores(ko, sv);
    const Scales sc = scales(s);
#pragma unroll
    for (int e = 0; e < 16; ++e) sv[e] = ok >> e & 1 ? sv[e] : -INFINITY;
    new_max(H, largest(sv, sc.ka, sc.kc));
    const float ms = m == -INFINITY ? 0.f : m;
    float p[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      // (selected once more: a scale of 0 times -inf is NaN)
      p[e] = ok >> e & 1 ? __builtin_amdgcn_exp2f(fmaf(sv[e], e < 8 ? sc.ka : sc.kc, -ms)) : 0.f;
      l += p[e];
    }
    uint4 ph[2], pl[2];
    operands(H, p, sc.va, sc.vc, ph, pl);
    values(buf & 1, vo);
    products(H, vo, ph, pl, sc.ua, sc.uc);
    if (s < 0 && bad_s) {
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
            const int d = 32 * y + 8 * (e >> 2) + 4 * h + (e & 3);
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
  if (tid == 0) base_s = kNoUnit;
  for (s0 = 0; s0 < ncache; s0 += SEG) {
    se = min(ncache, s0 + SEG);
    __syncthreads();
    // (12 more than the segment's: the loads run five stages past its end)
    for (int i = tid; i < min(2 * (se - s0) + 12, 2 * SEG + 12); i += 64 * W) {
      const int id = min(max(a.page_table[(size_t)b * a.max_pages + p0 + min(2 * s0 + i, np - 1)], 0), a.num_pages - 1);
      id_s[i] = id;
      if (KVT == 2) {
        ksc_s[i] = a.ksc[(size_t)id * a.nkv + j] * rs;
        const float v = a.vsc[(size_t)id * a.nkv + j];
        vsc_s[i] = v;
        if (v > 0.f && v < INFINITY) atomicMax(&base_s, (int)(__float_as_uint(v) >> 23) - 127);
      }
    }
    if (KVT == 2) {
      // A value scale is a factor on the page's weights and a power of two, the largest unit where that leaves
      // a factor in [2^-3, 2), since acc moves whenever the unit changes.
      __syncthreads();
      const int base = base_s;
      for (int i = tid; i < min(2 * (se - s0) + 12, 2 * SEG + 12); i += 64 * W) {
        const float v = vsc_s[i];
        int e = v > 0.f && v < INFINITY ? (int)(__float_as_uint(v) >> 23) - 127 : kNoUnit;
        e = e < base - 3 && e != kNoUnit ? max(e, base - kUnits) : max(base, -126);
        vsc_s[i] = ldexpf(v, -e);
        vex_s[i] = e;
      }
    }
    __syncthreads();
    // Keys run a stage ahead of values: while stage s is turned into weights (vector instructions), the
    // matrix cores form the scores of stage s + 1. In flight beyond that: keys of the next two stages, and
    // values.
    Half k0, k1, v0, v1;
    if constexpr (ROLES) {
      load_own(s0, k0);
      load_own(s0 + 1, k1);
      store_own(s0, k0);
      load_own(s0 + 2 - role, k0);
      store_own(s0 + 1, k1);
      load_own(s0 + 3 - role, k1);
    } else {
      load_keys(s0, k0);
      load_values(s0, v0);
      load_keys(s0 + 1, k1);
      load_values(s0 + 1, v1);
      store_keys(s0, k0);
      store_values(s0, v0);
      load_keys(s0 + 2, k0);
      store_keys(s0 + 1, k1);
      load_values(s0 + 2, v0);
      load_keys(s0 + 3, k1);
    }
    __syncthreads();
    floatx16 sv;
    if (busy) {
      uint4 ko[KS];
      keys(s0 & 1, ko);
      scores(ko, sv);
    }
    __syncthreads();
    const int end = min(se, nfull);
    auto step = [&](int s, Half &kr, Half &vr) {
      // (key buffer s & 1 is free: its scores were formed a step ago)
      auto stage = [&] {
        if constexpr (ROLES) {
          store_own(s + 2 - role, kr);
          load_own(s + 4 - role, kr);
          return;
        }
        store_keys(s + 2, kr);
        store_values(s + 1, vr);
        load_keys(s + 4, kr);
        load_values(s + 3, vr);
      };
      if (busy) {
        const Scales sc = scales(s);
        new_max(Cached(), largest(sv, sc.ka, sc.kc));
        const float ms = KVT != 2 && m == -INFINITY ? 0.f : m;  // (all scores -inf so far; fp8 keys are finite)
        float p[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(sv[e], e < 8 ? sc.ka : sc.kc, -ms));
          l += p[e];
        }
        uint4 ph[2], pl[2], ko[KS], vo[2][NT];
        keys((s + 1) & 1, ko);
        scores(ko, sv);
        stage();
        operands(Cached(), p, sc.va, sc.vc, ph, pl);
        values(s & 1, vo);
        products(Cached(), vo, ph, pl, sc.ua, sc.uc);
      } else {
        stage();
      }
      __syncthreads();
    };
    int s = s0;
    for (; s + 1 < end; s += 2) {
      step(s, k0, v1);
      step(s + 1, k1, v0);
    }
    if (s < end) step(s, k0, v1);
    if (end < se && busy)  // the candidate's last pair (in its buffers since the steps before)
      compute_masked(Cached(), end, end, own_bits((1u << (L - (p0 + 2 * end) * kPage)) - 1u), -1);
  }
  if (KVT == 1) {
    float z[4] = {0.f, 0.f, 0.f, 0.f};  // NaN where a sum is not finite
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) z[e & 3] = fmaf(acc[t][e], 0.f, z[e & 3]);
    if (__any((z[0] + z[1]) + (z[2] + z[3]) != 0.f)) {
      Special<NT * 16> sp;
      for (int i = 0; i < np; ++i) {
        const int id = min(max(a.page_table[(size_t)b * a.max_pages + p0 + i], 0), a.num_pages - 1);
        sp.template look<D>((const uint16_t *)a.vp + ((size_t)id * a.nkv + j) * (kPage * D), min(kPage, L - (p0 + i) * kPage),
                            lane, [&](int y) { return 8 * (y >> 2) + 4 * h + (y & 3); });
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] = sp.mend(acc[t][e], 16 * t + e);
    }
  }
  if (HALF) {  // from here on as over bf16 caches: weights below 1, acc in units of 1
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[t][e] = ldexpf(acc[t][e], unit - 12);
    unit = 0;
    m += 12.f;
    l *= 0x1p-12f;
  }
  // (the column once more, from the lane's number: held over the loop it would take registers that are not there)
  const Column my = column(__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)));
  const int tok = my.tok, head = my.head;
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
      compute_masked(Drafted(), -1, 0, own_bits(bits), t0);
    }
  }
  if (!my.present) return;
  {
    const uint32_t u = __float_as_uint(l);
    const auto t = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    l = __uint_as_float(t[0]) + __uint_as_float(t[1]);
  }
  const int64_t row = tr.r0 + tok, at = ((int64_t)(part_row(a, b, tr) + tok) * a.nq + head) * a.slots + c;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 32 * t + 8 * i + 4 * h;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = nc == 1 ? acc[t][4 * i + e] * inv : acc[t][4 * i + e];
      if (nc == 1) store4((T *)a.o + row * a.os + (int64_t)head * D + d, v);
      else store4(a.pacc + at * D + d, v);
    }
  if (nc > 1 && h == 0) a.pml[at] = make_float2(m, l);
}

// Joins the chunks of drafted tokens' q-heads, N of them to a wave: weights 2^(m - M) from one load
// per lane (at most 64 chunks), then the chunk sums in order, two chunks at a time (one per half of the
// wave, 16 or 8 bytes a lane) and four such pairs in flight. N = 2 where that keeps the grid in one round
// (the wave is one chain of memory round trips, whatever it does beside): 14336 q-heads of 4 chunks of 128
// dims, 29 MB read, in 9 us; 256 of 10 chunks in 4.
template <int D, int N, typename T>
__global__ __launch_bounds__(256) void k_tree_merge(TreeArgs a) {
  const int b = blockIdx.y, lane = threadIdx.x & 63, half = lane >> 5;
  const int item = N * __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (threadIdx.x >> 6));
  const TreeRows tr = tree_rows(a, b);
  const int nc = tree_split(a, tr).chunks, items = tr.n * a.nq;
  if (item >= items || nc == 1) return;
  constexpr int E = D / 32;
  typedef float vec __attribute__((ext_vector_type(E)));
  const vec *p[N];
  float2 ml[N];
  vec x[N][4];
#pragma unroll
  for (int z = 0; z < N; ++z) {
    const int64_t at = ((int64_t)part_row(a, b, tr) * a.nq + min(item + z, items - 1)) * a.slots;
    p[z] = (const vec *)(a.pacc + at * D) + (lane & 31);
    ml[z] = lane < nc ? a.pml[at + lane] : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int u = 0; u < 4; ++u) x[z][u] = p[z][(size_t)min(2 * u + half, nc - 1) * 32];
  }
#pragma unroll
  for (int z = 0; z < N; ++z) {
    const float M = wmax(ml[z].x);
    const float f = ml[z].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[z].x - M);
    const float l = wsum(f * ml[z].y);
    vec v = {};
    for (int i = 0; i < nc; i += 8) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int k = i + 2 * u;
        const float w0 = lane_value(f, min(k, 63)), w1 = lane_value(f, min(k + 1, 63));
        const float w = half ? w1 : w0;
        if (k + half < nc) v += w * x[z][u];
        if (i + 8 < nc) x[z][u] = p[z][(size_t)min(k + 8 + half, nc - 1) * 32];
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const uint32_t u = __float_as_uint(v[e]);
      const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
      v[e] = (__uint_as_float(r[0]) + __uint_as_float(r[1])) * inv;
    }
    if (half || item + z >= items) continue;
    const int t = (item + z) / a.nq, head = item + z - t * a.nq;
    T *o = (T *)a.o + (tr.r0 + t) * a.os + (int64_t)head * D + lane * E;
    if constexpr (sizeof(T) == 4) {
      *(vec *)o = v;
    } else {
      uint32_t y[E / 2], lo;
#pragma unroll
      for (int e = 0; e < E; e += 2) split2(v[e], v[e + 1], y[e / 2], lo);
      if constexpr (E == 4) *(uint2 *)o = make_uint2(y[0], y[1]);
      else *(uint32_t *)o = y[0];
    }
  }
}

// ------------------------------------------------------------------------------- launch

struct TreePlan {
  bool wide;   // k_tree_wide
  int nc;      // column tiles of a k_tree block
  int cols;    // columns of a block
  int blocks;  // column blocks of the longest draft
  int fill;    // (chunk, kv-head) pairs that fill the chip
  int unit;    // pages that chunks are multiples of
  int draft_tokens, draft_pages;
  int least;   // pages of the shortest chunk that is worth a block
  int slots;   // chunk slots
};

constexpr int kWideWaves = 4;

// Drafted tokens there can be (an array may have rows to spare).
static int64_t draft_rows(const kvprm_batch &b, const kvprm_tree &t) {
  return min((int64_t)b.batch * t.max_rows, t.num_rows);
}
static int draft_extra(const TreePlan &p, int n) { return (n + p.draft_tokens - 1) / p.draft_tokens * p.draft_pages; }

// Blocks that fill the chip (see tree_plan).
static int full_chip(const Dims &dm, bool wide) { return wide && dm.d == 64 ? 768 : 512; }

// Kernel by the longest draft's columns where the chip is full (launch_tree has the rule for fewer blocks): k_tree
// up to 32, which a wave holds at once, else k_tree_wide. At 17 to 32 columns k_tree took 13.9 us and k_tree_wide 16.6
// (1103 tokens, 32 columns; 12.0 in blocks of 16), 25.5 and 30.2 (24 fp8 caches of 4800, 32 columns), 91.0 and 88.6 (8
// caches of 16384 to 32768, 28 columns); at 33 to 64, where k_tree reads the pages twice, 42.1 and 34.2 (the 24 caches,
// 48 columns), 108 and 95 (the 8, 56 columns). Left at 32 columns: 16 x 4000 bf16 tokens, 67.4 us, would take 62.6 in
// k_tree_wide.
// Chunks leave as many blocks as the chip takes: two of k_tree_wide on a compute unit (three at d_h = 64), which are
// resident at once. Fewer or more both lose: 24 ragged fp8 caches, d_h = 64, 52.0 us at 680 blocks, 49.6 at 768, 58.2
// at 1024; 8 long bf16 caches, d_h = 128, 402 us at 400, 332 at 512, 399 at 600. Two of k_tree as well; they are
// resident at once but for 32 columns at d_h = 128 and fp32 rows over bf16 caches there, whose registers leave room for
// one block: 256, 512 and 1024 blocks take 29.2, 25.5 and 29.9 us (24 fp8 caches of 4800, 32 columns, d_h = 64), 91.3,
// 90.8 and 108 (8 long bf16 caches, 28 columns, d_h = 128), 68.2, 76.8 and 96.8 (16 x 4096 bf16 tokens, 112
// columns, d_h = 128, which k_tree_wide takes). Column blocks are counted by the average draft, draft_rows / batch,
// since a candidate's missing ones are no blocks. A k_tree_wide chunk has 16 pages or more: 24 x 1200 tokens, 96
// columns, take 25.2, 23.8 and 26.9 us with least chunks of 8, 16 and 32 pages. Drafted tokens count as pages of the
// last chunk (4 for 32 tokens of k_tree_wide, a unit for 64 of k_tree): 12.1 us instead of 13.9 for 1103 tokens, 326
// instead of 330 on the long caches; 2 to 8 pages are alike there. Chunk slots: what fills the chip eight times over if
// the batch's candidates were all as long as the table.
// 4-bit caches: k_tree has 16 columns a block at d_h = 128 (two tiles beside widened keys and values leave the
// registers of one wave a unit, or of two that wait for each other's conversions) and where 32 would not hold the
// draft. Reading a page once more costs little there. Blocks of 32 and of 16 columns, us, bf16 rows: 8 caches of
// 16384 to 32768 tokens, 28 columns, 54 / 48; 16 of 4000, 32 columns, 39 / 35; 64 of 2000, 28 columns, 42 / 32; 8 of
// 8000, 2 drafted of 16 heads, 25 / 19; 16 of 300, 64 columns (k_tree_wide / 16), 23 / 13; fp32 rows: the first 70 /
// 57, the second 55 / 43, 29 of 75 tokens, 304 columns, 124 / 89. d_h = 64, up to 32 columns: 24 of 4800, 23.6 / 28.2
// (fp32 rows 27.1 / 30.2), but 64 of 3000, 28 columns, 32.3 / 29.6; more, fp32 rows: 16 of 500, 128 columns, 20.8 /
// 11.8, 24 of 1 to 9000, 4 to 192 columns, 74.4 / 78.7. (More blocks of 16 instead of k_tree_wide, up to 1024: 24 of
// 3000 to 6000, 160 columns, d_h = 64, 68 -> 77, 12 of 8000, 336 columns, d_h = 128, 137 -> 164.)
static TreePlan tree_plan(const Dims &dm, const kvprm_batch &b, const kvprm_tree &t, bool wide) {
  TreePlan p;
  const int cols = t.max_rows * dm.g;
  p.wide = wide;
  p.nc = cols <= 16 || (dm.kvdt == 3 && (dm.d == 128 || cols > 32)) ? 1 : 2;
  p.cols = p.wide ? 32 * kWideWaves : 16 * p.nc;
  p.blocks = (cols + p.cols - 1) / p.cols;
  // Spread evenly, unless the average draft needs fewer blocks than the longest: 24 drafts of 1 to 48 tokens of
  // 4 query heads took 55 us in blocks of 128 columns and 68 in blocks of 96.
  const int64_t rows = draft_rows(b, t);
  if (p.wide && rows * dm.g > (int64_t)b.batch * (p.blocks - 1) * p.cols)
    p.cols = ((cols + p.blocks - 1) / p.blocks + 31) / 32 * 32;
  // average column blocks of a candidate, in 16ths
  const int64_t avg = max((int64_t)16, min((int64_t)p.blocks * 16, rows * dm.g * 16 / b.batch / p.cols + 8));
  p.fill = (int)max((int64_t)1, full_chip(dm, p.wide) * 16 / avg);
  // (fp32 caches: a wave takes pages, not pairs; units of 8 pages took 11.4 us for 4 x 512 tokens, of 4 11.0)
  p.unit = p.wide ? 2 : dm.kvdt == 0 ? kTreeWaves : 2 * kTreeWaves;
  p.least = p.wide ? 16 : p.unit;
  p.draft_tokens = p.wide ? 32 : 64;
  p.draft_pages = p.wide ? 4 : p.unit;
  const int64_t items = (int64_t)b.batch * dm.nkv;
  int64_t slots = (8 * p.fill + items - 1) / items;
  slots = min(slots, (int64_t)draft_chunks(b.max_pages, draft_extra(p, t.max_rows), p.least));
  p.slots = (int)max((int64_t)1, min(slots, (int64_t)64));
  return p;
}

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

static bool may_be_wide(const Dims &dm, const kvprm_tree &t) {
  return t.dtype == KVPRM_BF16 && dm.kvdt != 0 && t.max_rows * dm.g > 32;
}

static size_t parts_bytes(const Dims &dm, int64_t parts) {  // parts: (row, slot) pairs
  return align256((size_t)parts * dm.nq * dm.d * 4) + align256((size_t)parts * dm.nq * 8);
}

// What one call takes.
size_t tree_ws_need(const Dims &dm, const kvprm_batch &b, const kvprm_tree &t) {
  int slots = tree_plan(dm, b, t, false).slots;
  if (may_be_wide(dm, t)) slots = max(slots, tree_plan(dm, b, t, true).slots);
  return slots == 1 ? 256 : parts_bytes(dm, draft_rows(b, t) * slots);
}

// What the largest call of at most so many candidates, pages, rows and rows per candidate takes, so that a workspace
// sized once serves smaller batches, whose chip is filled by more chunks. With r = draft_rows, B candidates and n
// kv-heads a plan has slots < 8 fill / (B n) + 1 and fill <= full 16 / avg, where avg >= 16 and avg >= r g 16 / (B cols):
// r slots <= r + 8 full / n min(r / B, cols / g), which grows with all four; nor are there more slots than
// chunks.
size_t tree_ws_bytes(const Dims &dm, const kvprm_batch &b, const kvprm_tree &t) {
  const int64_t rows = draft_rows(b, t);
  int64_t parts = 0;
  for (int wide = 0; wide <= may_be_wide(dm, t); ++wide) {
    const TreePlan p = tree_plan(dm, b, t, wide);
    const int64_t chunks = min((int64_t)64, (int64_t)draft_chunks(b.max_pages, draft_extra(p, t.max_rows), p.least));
    const int64_t columns = wide ? 32 * kWideWaves : 32;
    const int64_t filled = 8 * (int64_t)full_chip(dm, wide) * min(t.max_rows * (int64_t)dm.g, columns);
    const int64_t per = dm.nkv * dm.g;
    if (chunks > 1) parts = max(parts, min(rows * chunks, rows + (filled + per - 1) / per));
  }
  return max((size_t)256, parts_bytes(dm, parts));
}

static int cached_pages(const kvprm_batch &b, int i) {
  return b.lengths_host ? (b.lengths_host[i] + kPage - 1) / kPage : b.max_pages;
}

// Most pages of a chunk: the fewest (multiples of p.unit, at least p.least) whose chunks leave the grid
// within p.fill blocks and each candidate within its slots.
static int tree_chunk_pages(const Dims &dm, const kvprm_batch &b, const kvprm_tree &t, const TreePlan &p) {
  int longest = 1;
  for (int i = 0; i < b.batch; ++i) longest = max(longest, cached_pages(b, i));
  longest += draft_extra(p, t.max_rows);
  const int extra = draft_extra(p, (int)(draft_rows(b, t) / b.batch));
  const int64_t most = max((int64_t)p.fill / dm.nkv, (int64_t)b.batch);
  // in units: the least is (too few or) enough, the longest candidate whole is enough
  int lo = max(p.least, (longest + p.slots - 1) / p.slots + p.unit - 1) / p.unit;
  int hi = max(lo, (longest + p.unit - 1) / p.unit);
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    int64_t chunks = 0;
    for (int i = 0; i < b.batch; ++i)
      chunks += draft_chunks(cached_pages(b, i), extra, mid * p.unit);
    if (chunks <= most) hi = mid;
    else lo = mid + 1;
  }
  return lo * p.unit;
}

hipError_t launch_tree(const Dims &dm, const kvprm_kv_cache &c, const kvprm_batch &b, int layer,
                       const kvprm_tree &t, void *ws, hipStream_t s) {
  TreePlan p = tree_plan(dm, b, t, false);
  int chunk_pages = tree_chunk_pages(dm, b, t, p);
  auto chunks_of = [&](int i) { return draft_chunks(cached_pages(b, i), draft_extra(p, t.max_rows), chunk_pages); };
  int64_t items = 0;  // chunks of all candidates
  for (int i = 0; i < b.batch; ++i) items += chunks_of(i);
  // Blocks of 16 columns (short chains, pages read once per block from the caches) while they leave the chip's
  // waves unfilled. Instead of 32 columns, up to 768 blocks: 1103 tokens, 32 columns (160 blocks) 13.9 -> 12.0 us,
  // 2 x 2500 (672 blocks) 25.0 -> 21.5, but 16 x 4000 (1024 blocks) 67.4 -> 73.4. Instead of k_tree_wide, up to
  // 512: 1103 tokens, 64 columns (320 blocks) 17.7 -> 14.6, 300 tokens, 128 columns (256) 19.3 -> 12.8, 4 x 700
  // fp8 tokens, 64 columns 16.1 -> 10.5, but 2500 tokens, 64 columns (over 512) 18.9 -> 20.9.
  const int64_t blocks16 = items * dm.nkv * ((t.max_rows * dm.g + 15) / 16);
  if (may_be_wide(dm, t) && blocks16 > 512) {
    p = tree_plan(dm, b, t, true);
    chunk_pages = tree_chunk_pages(dm, b, t, p);
  } else if (blocks16 <= 768) {
    p.nc = 1;
    p.cols = 16;
    p.blocks = (t.max_rows * dm.g + 15) / 16;
  }
  const size_t tiles = (size_t)c.num_pages * dm.nkv;
  const size_t bytes = tiles * tile_bytes(dm.kvdt, dm.d);
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
  a.chunk_pages = chunk_pages;
  a.unit = p.unit;
  a.draft_tokens = p.draft_tokens, a.draft_pages = p.draft_pages;
  a.block_cols = p.cols;
  a.slots = p.slots;
  a.pacc = (float *)ws;
  a.part_rows = draft_rows(b, t) < t.num_rows ? t.max_rows : 0;
  a.pml = (float2 *)((char *)ws + align256((size_t)draft_rows(b, t) * dm.nq * p.slots * dm.d * 4));
  int chunks = 1;
  items = 0;
  for (int i = 0; i < b.batch; ++i) {
    chunks = max(chunks, chunks_of(i));
    items += chunks_of(i);
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
  hipLaunchKernelGGL((k_tree_wide<K_, D_, kWideWaves>), grid, dim3(64 * kWideWaves), 0, s, a)
  if (p.wide) {
    if (dm.kvdt == 1 && dm.d == 64) { KVPRM_WIDE(1, 64); }
    else if (dm.kvdt == 1) { KVPRM_WIDE(1, 128); }
    else if (dm.kvdt == 3 && dm.d == 64) { KVPRM_WIDE(3, 64); }
    else if (dm.kvdt == 3) { KVPRM_WIDE(3, 128); }
    else if (dm.d == 64) { KVPRM_WIDE(2, 64); }
    else { KVPRM_WIDE(2, 128); }
  } else if (dm.kvdt == 0) { KVPRM_TREE_D(0) }
  else if (dm.kvdt == 1) { KVPRM_TREE_D(1) }
  else if (dm.kvdt == 3) {
    if (dm.d == 64) { KVPRM_TREE_T(3, 64) }
    else if (bf16) { KVPRM_TREE(3, 128, 1, uint16_t); }  // (see tree_plan)
    else { KVPRM_TREE(3, 128, 1, float); }
  }
  else { KVPRM_TREE_D(2) }
#undef KVPRM_WIDE
#undef KVPRM_TREE_D
#undef KVPRM_TREE_T
#undef KVPRM_TREE_N
#undef KVPRM_TREE
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || chunks == 1) return e;
  // (8192 waves are resident at once)
  const int n = draft_rows(b, t) * dm.nq > 8192 ? 2 : 1;
  const dim3 mgrid((unsigned)(((int64_t)t.max_rows * dm.nq + 4 * n - 1) / (4 * n)), b.batch);
#define KVPRM_MERGE_T(D_, N_)                                                                     \
  if (bf16) hipLaunchKernelGGL((k_tree_merge<D_, N_, uint16_t>), mgrid, dim3(256), 0, s, a);      \
  else hipLaunchKernelGGL((k_tree_merge<D_, N_, float>), mgrid, dim3(256), 0, s, a)
#define KVPRM_MERGE(D_)                    \
  if (n == 1) { KVPRM_MERGE_T(D_, 1); }    \
  else { KVPRM_MERGE_T(D_, 2); }
  if (dm.d == 64) { KVPRM_MERGE(64) }
  else { KVPRM_MERGE(128) }
#undef KVPRM_MERGE_T
#undef KVPRM_MERGE
  return hipGetLastError();
}

}  // namespace kvprm
