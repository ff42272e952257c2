// Device helpers shared by the attention kernels over the paged cache (kvprm_attn.hip,
// kvprm_tree.hip): a page pair's tiles from memory to matrix-core operands.
#pragma once

#include "kvprm_mx_common.h"

namespace kvprm {

template <bool HIGH>
__device__ __forceinline__ uint32_t fp8x2_to_bf16x2(uint32_t word) {
  // two OCP e4m3 codes (bytes 0, 1 or 2, 3) -> two bf16 in one instruction; every e4m3 value is
  // a bf16 value and the scale is 1, so the conversion is exact
  typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
  const bf16x2v v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, 1.0f, HIGH);
  return __builtin_bit_cast(uint32_t, v);
}

// Lane i's value of v, for a wave-uniform i (a scalar read of one lane: no LDS round trip).
__device__ __forceinline__ int lane_value(int v, int i) { return __builtin_amdgcn_readlane(v, i); }
__device__ __forceinline__ float lane_value(float v, int i) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), i));
}

// Raw registers of one page pair of one kv-head, in tile byte order (16 bytes per lane and
// instruction): K tiles of pages A and B, then their V tiles. bf16 uses D/32 of each, fp8 D/64.
template <int D>
struct PairRaw {
  uint4 k[2][D / 32];
  uint4 v[2][D / 32];
};

// The same of a 4-bit cache: a lane has D / 8 bytes of each tile's codes (in the low words of 16), its byte
// of the keys' scales and the D / 8 scales of its values' slots.
template <int D>
struct PairRaw4 {
  uint4 k[2], v[2], vs[2];
  uint32_t ks[2];
};
template <int KVT, int D>
using PairOf = std::conditional_t<KVT == 3, PairRaw4<D>, PairRaw<D>>;

// Loads a pair from tile base pointers: global memory read once (STREAM, non-temporal), or LDS.
template <int KVT, int D, bool STREAM>
__device__ __forceinline__ void load_pair_raw(const uint4 *kA, const uint4 *kB, const uint4 *vA,
                                              const uint4 *vB, int lane, PairRaw<D> &r) {
  constexpr int N = KVT == 1 ? D / 32 : D / 64;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (STREAM) {
      r.k[0][i] = ld_stream(kA + i * 64 + lane);
      r.k[1][i] = ld_stream(kB + i * 64 + lane);
      r.v[0][i] = ld_stream(vA + i * 64 + lane);
      r.v[1][i] = ld_stream(vB + i * 64 + lane);
    } else {
      r.k[0][i] = kA[i * 64 + lane];
      r.k[1][i] = kB[i * 64 + lane];
      r.v[0][i] = vA[i * 64 + lane];
      r.v[1][i] = vB[i * 64 + lane];
    }
  }
}

// Raw pair -> bf16 MFMA operands. K: lane holds token lane % 16, 8 dims per 32-dim block
// (bf16: dims 32kk + 8c + i; fp8: dims 16 (4 (kk/2) + c) + 8 (kk%2) + i). V (tile stores 4
// consecutive slots of r dims 16 apart): VA[nb] = slots 4c..4c+3 of dim 16 nb + lane % 16.
template <int KVT, int D>
__device__ __forceinline__ void unpack_pair(const PairRaw<D> &r, uint4 *KA, uint4 *KB, uint2 *VA,
                                            uint2 *VB) {
  constexpr int NKB = D / 32, NDB = D / 16;
  if (KVT == 1) {
#pragma unroll
    for (int kk = 0; kk < NKB; ++kk) {
      KA[kk] = r.k[0][kk];
      KB[kk] = r.k[1][kk];
    }
#pragma unroll
    for (int q2 = 0; q2 < NDB / 2; ++q2) {
      VA[2 * q2] = make_uint2(r.v[0][q2].x, r.v[0][q2].y);
      VA[2 * q2 + 1] = make_uint2(r.v[0][q2].z, r.v[0][q2].w);
      VB[2 * q2] = make_uint2(r.v[1][q2].x, r.v[1][q2].y);
      VB[2 * q2 + 1] = make_uint2(r.v[1][q2].z, r.v[1][q2].w);
    }
  } else {
#pragma unroll
    for (int kp = 0; kp < NKB / 2; ++kp) {
      const uint4 ra = r.k[0][kp], rb = r.k[1][kp];
      KA[2 * kp] = make_uint4(fp8x2_to_bf16x2<false>(ra.x), fp8x2_to_bf16x2<true>(ra.x),
                              fp8x2_to_bf16x2<false>(ra.y), fp8x2_to_bf16x2<true>(ra.y));
      KA[2 * kp + 1] = make_uint4(fp8x2_to_bf16x2<false>(ra.z), fp8x2_to_bf16x2<true>(ra.z),
                                  fp8x2_to_bf16x2<false>(ra.w), fp8x2_to_bf16x2<true>(ra.w));
      KB[2 * kp] = make_uint4(fp8x2_to_bf16x2<false>(rb.x), fp8x2_to_bf16x2<true>(rb.x),
                              fp8x2_to_bf16x2<false>(rb.y), fp8x2_to_bf16x2<true>(rb.y));
      KB[2 * kp + 1] = make_uint4(fp8x2_to_bf16x2<false>(rb.z), fp8x2_to_bf16x2<true>(rb.z),
                                  fp8x2_to_bf16x2<false>(rb.w), fp8x2_to_bf16x2<true>(rb.w));
    }
#pragma unroll
    for (int q4 = 0; q4 < NDB / 4; ++q4) {
      const uint32_t wa[4] = {r.v[0][q4].x, r.v[0][q4].y, r.v[0][q4].z, r.v[0][q4].w};
      const uint32_t wb[4] = {r.v[1][q4].x, r.v[1][q4].y, r.v[1][q4].z, r.v[1][q4].w};
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        VA[4 * q4 + jj] = make_uint2(fp8x2_to_bf16x2<false>(wa[jj]), fp8x2_to_bf16x2<true>(wa[jj]));
        VB[4 * q4 + jj] = make_uint2(fp8x2_to_bf16x2<false>(wb[jj]), fp8x2_to_bf16x2<true>(wb[jj]));
      }
    }
  }
}

// ---- 4-bit tiles (layout: see kvprm_kv_cache)

// Products of a query in several terms give scores times 2^-32, so that terms of unlike sign do not overflow on the way to
// a score that does (an infinity of each sign would be a NaN): a stored key can be as large as fp32's range. What
// is left of a value, times log2(e) / sqrt(d_h), below 2^-95 is lost.
constexpr int kScoreShift4 = 32;
constexpr float kScoreUnit4 = 4294967296.f;

// N = 8 or 16 bytes into the low words of 16.
template <int N, bool STREAM>
__device__ __forceinline__ uint4 load_bytes(const char *p) {
  if constexpr (N == 16) return STREAM ? ld_stream((const uint4 *)p) : *(const uint4 *)p;
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 v = STREAM ? __builtin_nontemporal_load((const u32x2 *)p) : *(const u32x2 *)p;
  return make_uint4(v.x, v.y, 0, 0);
}
// This lane's place in a tile: K codes of dims D / 4 (lane / 16) .. of slot lane % 16, and their scale (the codes
// of 32 dims of a slot are 16 bytes, so at D = 64 a lane takes half of them).
template <int D>
__device__ __forceinline__ uint32_t key_code4(int lane) {
  return D == 128 ? 16 * lane : ((lane >> 5) * 16 + (lane & 15)) * 16 + (lane >> 4 & 1) * 8;
}
template <int D>
__device__ __forceinline__ uint32_t key_scale4(int lane) {
  return 8 * D + (D == 128 ? lane : (lane >> 5) * 16 + (lane & 15));
}
// V codes of slots 4 (lane / 16) .. of dims lane % 16 + 16 i, and the scales of these slots.
template <int D>
__device__ __forceinline__ uint32_t value_code4(int lane) { return lane * (D / 8); }
template <int D>
__device__ __forceinline__ uint32_t value_scale4(int lane) { return 8 * D + (lane >> 4) * (D / 8); }

template <int D, bool STREAM>
__device__ __forceinline__ void load_pair_raw4(const char *kA, const char *kB, const char *vA, const char *vB,
                                               int lane, PairRaw4<D> &r) {
  constexpr int N = D / 8;
  r.k[0] = load_bytes<N, STREAM>(kA + key_code4<D>(lane));
  r.k[1] = load_bytes<N, STREAM>(kB + key_code4<D>(lane));
  r.ks[0] = *(const uint8_t *)(kA + key_scale4<D>(lane));
  r.ks[1] = *(const uint8_t *)(kB + key_scale4<D>(lane));
  r.v[0] = load_bytes<N, STREAM>(vA + value_code4<D>(lane));
  r.v[1] = load_bytes<N, STREAM>(vB + value_code4<D>(lane));
  r.vs[0] = load_bytes<N, false>(vA + value_scale4<D>(lane));
  r.vs[1] = load_bytes<N, false>(vB + value_scale4<D>(lane));
}

// Two e2m1 codes (byte B of w) -> two bf16, times a power of two. The instruction takes the exponent of `scale` alone,
// whatever its sign and significand; the product is exact up to 2^125, and an exponent of all ones (scale byte 255)
// gives NaN.
template <int B>
__device__ __forceinline__ uint32_t fp4x2_to_bf16x2(uint32_t w, float scale) {
  typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
  const bf16x2v v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B);
  return __builtin_bit_cast(uint32_t, v);
}
// A float whose exponent is byte B of w (a scale's biased exponent), for the conversions: other bits are w's.
template <int B>
__device__ __forceinline__ float scale_of(uint32_t w) {
  return __uint_as_float(B == 3 ? w >> 1 : w << (23 - 8 * B));
}
// The codes of 8 dims of a slot -> bf16.
__device__ __forceinline__ uint4 keys4(uint32_t w, float scale) {
  return make_uint4(fp4x2_to_bf16x2<0>(w, scale), fp4x2_to_bf16x2<1>(w, scale),
                    fp4x2_to_bf16x2<2>(w, scale), fp4x2_to_bf16x2<3>(w, scale));
}
// The codes of 4 slots of dims m and m + 16 (a byte each, with the slots' scales) -> the slots of m, those of m + 16.
// The two codes of a byte share their scale, so that one instruction converts them; two more per pair of slots
// bring a dim's slots side by side, as the products want them.
__device__ __forceinline__ void values4(uint32_t w, uint32_t scales, uint2 &lo, uint2 &hi) {
  const uint32_t x0 = fp4x2_to_bf16x2<0>(w, scale_of<0>(scales)), x1 = fp4x2_to_bf16x2<1>(w, scale_of<1>(scales));
  const uint32_t x2 = fp4x2_to_bf16x2<2>(w, scale_of<2>(scales)), x3 = fp4x2_to_bf16x2<3>(w, scale_of<3>(scales));
  lo = make_uint2(__builtin_amdgcn_perm(x1, x0, 0x05040100u), __builtin_amdgcn_perm(x3, x2, 0x05040100u));
  hi = make_uint2(__builtin_amdgcn_perm(x1, x0, 0x07060302u), __builtin_amdgcn_perm(x3, x2, 0x07060302u));
}
__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Raw pair -> operands as unpack_pair gives them; K: dims D / 4 (lane / 16) + 8 kk + i of token lane % 16.
template <int D>
__device__ __forceinline__ void unpack_pair4(const PairRaw4<D> &r, uint4 *KA, uint4 *KB, uint2 *VA, uint2 *VB) {
  const float sa = scale_of<0>(r.ks[0]), sb = scale_of<0>(r.ks[1]);
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk) {
    KA[kk] = keys4(word(r.k[0], kk), sa);
    KB[kk] = keys4(word(r.k[1], kk), sb);
    values4(word(r.v[0], kk), word(r.vs[0], kk), VA[2 * kk], VA[2 * kk + 1]);
    values4(word(r.v[1], kk), word(r.vs[1], kk), VB[2 * kk], VB[2 * kk + 1]);
  }
}

// The dims that a lane's K operand of 32-dim block kk starts at (lane / 16 = c).
template <int KVT, int D>
__device__ __forceinline__ int key_dim(int kk, int c) {
  return KVT == 1 ? kk * 32 + 8 * c : KVT == 2 ? 16 * (4 * (kk >> 1) + c) + 8 * (kk & 1) : D / 4 * c + 8 * kk;
}

// A pair's tiles from tile base addresses to registers, and from there to operands, by cache type.
template <int KVT, int D, bool STREAM>
__device__ __forceinline__ void load_pair_of(const char *kA, const char *kB, const char *vA, const char *vB, int lane,
                                             PairOf<KVT, D> &r) {
  if constexpr (KVT == 3)
    load_pair_raw4<D, STREAM>(kA, kB, vA, vB, lane, r);
  else
    load_pair_raw<KVT, D, STREAM>((const uint4 *)kA, (const uint4 *)kB, (const uint4 *)vA, (const uint4 *)vB, lane, r);
}
template <int KVT, int D>
__device__ __forceinline__ void unpack_pair_of(const PairOf<KVT, D> &r, uint4 *KA, uint4 *KB, uint2 *VA, uint2 *VB) {
  if constexpr (KVT == 3)
    unpack_pair4<D>(r, KA, KB, VA, VB);
  else
    unpack_pair<KVT, D>(r, KA, KB, VA, VB);
}

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int lane_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row shifts by 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row 0 into 1, 2 into 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // rows 0 and 1 into 2 and 3
  return v;
}

}  // namespace kvprm
