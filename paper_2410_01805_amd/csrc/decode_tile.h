// Pieces of the decode kernels (one new token per sequence: decode.hip, paged_decode.hip): reductions over the quarters of a wavefront
// and the matrix-core form of 32 keys of a wavefront.
#pragma once
#include "attn_common.h"

namespace locret {

typedef float dec_f32x4 __attribute__((ext_vector_type(4)));

// the upper halves of a and b as one word, a's low
__device__ __forceinline__ uint32_t upper_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t lower_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

// max and sum over the four lanes lane % 16, + 16, + 32, + 48, in all of them: after a swap one register holds one half's value
// in both halves and the other the other's
__device__ __forceinline__ float max_across_quarters(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return max_across_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_across_quarters(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t w = __float_as_uint(__uint_as_float(r[0]) + __uint_as_float(r[1]));
  const auto t = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

// N consecutive words, 4-byte aligned
typedef uint32_t dec_u32x3 __attribute__((ext_vector_type(3), aligned(4)));
template <int N> __device__ __forceinline__ void load_words(const void* p, uint32_t* w) {
  if constexpr (N == 4) { const uint4 v = *(const uint4*)p; w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
  else if constexpr (N == 3) { const dec_u32x3 v = *(const dec_u32x3*)p; w[0] = v[0]; w[1] = v[1]; w[2] = v[2]; }
  else if constexpr (N == 2) { const uint2 v = *(const uint2*)p; w[0] = v.x; w[1] = v.y; }
  else w[0] = *(const uint32_t*)p;
}

// 32 keys of one wavefront for S^T = K Q^T and O = P V with v_mfma_f32_16x16x32_bf16, straight from memory to registers.  Lane (n = lane % 16, kg = lane / 16):
//   ka[b][ks]  16 bytes of key 8 (n / 4) + 4 b + n % 4 from dim 32 ks + 8 kg: rows of the A operand of block b of
//              S^T = K Q^T, ordered so that the lane's accumulators, rows 4 kg + r of the two blocks, are its keys 8 kg + 4 b + r
//   vw[r]      dims n NV .. n NV + NV - 1 of key 8 kg + r
template <int D> struct DecTile {
  static constexpr int NKS = D / 32, NV = D / 16, PARTS = 3;
  bf16x8 ka[2][NKS];
  uint32_t vw[8][NV / 2];
  // (keys from k1 on repeat the last one; kb is the same in the whole wavefront, so only the offsets inside the block are per lane)
  __device__ __forceinline__ void load_k(const bf16_t* Kb, int kb, int k1) {
    const int n = threadIdx.x & 15, kg = (threadIdx.x & 63) >> 4, last = k1 - 1 - kb;
    const bf16_t* base = Kb + (int64_t)kb * D;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int off = min(8 * (n >> 2) + (n & 3) + 4 * b, last) * D + kg * 8;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) ka[b][ks] = *(const bf16x8*)(base + off + ks * 32);
    }
  }
  __device__ __forceinline__ void load_v(const bf16_t* Vb, int kb, int k1) {
    const int n = threadIdx.x & 15, kg = (threadIdx.x & 63) >> 4, last = k1 - 1 - kb;
    const bf16_t* base = Vb + (int64_t)kb * D;
#pragma unroll
    for (int r = 0; r < 8; ++r) load_words<NV / 2>(base + (min(8 * kg + r, last) * D + n * NV), vw[r]);
  }
  // the rows that repeat the last one: zeros, an infinite value times a probability of 0 would reach the output
  __device__ __forceinline__ void clear_v(int kb, int k1) {
    const int over = 8 * (int)((threadIdx.x & 63) >> 4) - (k1 - 1 - kb);
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int w = 0; w < NV / 2; ++w) vw[r][w] = over + r > 0 ? 0u : vw[r][w];
  }
  __device__ __forceinline__ void logits(const bf16x8 (&qb)[NKS], dec_f32x4 (&s)[2]) const {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      s[b] = dec_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[b][ks], qb[ks], s[b], 0, 0, 0);
    }
  }
  // o[i] += P V for dims n NV + i, n = 0..15: the B operand of dim i is the eight keys' values of that dim, taken two keys at
  // a time from the rows' words
  __device__ __forceinline__ void accumulate(bf16x8 p, dec_f32x4 (&o)[NV]) const {
#pragma unroll
    for (int w = 0; w < NV / 2; ++w) {
      const uint4 lo = make_uint4(lower_halves(vw[0][w], vw[1][w]), lower_halves(vw[2][w], vw[3][w]),
                                  lower_halves(vw[4][w], vw[5][w]), lower_halves(vw[6][w], vw[7][w]));
      const uint4 hi = make_uint4(upper_halves(vw[0][w], vw[1][w]), upper_halves(vw[2][w], vw[3][w]),
                                  upper_halves(vw[4][w], vw[5][w]), upper_halves(vw[6][w], vw[7][w]));
      o[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, __builtin_bit_cast(bf16x8, lo), o[2 * w], 0, 0, 0);
      o[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, __builtin_bit_cast(bf16x8, hi), o[2 * w + 1], 0, 0, 0);
    }
  }
};

}  // namespace locret
