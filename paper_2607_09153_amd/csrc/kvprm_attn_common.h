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
