// 32 keys of a wavefront from pages to registers, in the layout of the operands of S^T = K Q^T and O = P V with up to 16 query rows on the other side.
#pragma once
#include "decode_tile.h"

namespace locret {

// DecTile's operands from two places: rows 0..15 and 16..31 of the tile (pages of 16 units; the same place for larger ones).
// SMALL: the two places differ.  Otherwise `lo` is the same in the whole wavefront and the lanes add 32-bit offsets to it.
template <bool SMALL> __device__ __forceinline__ const void* tile_row(const void* lo, const void* hi, bool second, uint32_t bytes) {
  if constexpr (SMALL) return (const char*)(second ? hi : lo) + bytes;
  else return (const char*)lo + bytes;
}
template <int D, bool SMALL> struct PagedTileBf16 : DecTile<D> {
  typedef DecTile<D> Base;
  static constexpr int NQ = Base::NKS;
  typedef bf16x8 q_t;
  __device__ __forceinline__ void load_k(const bf16_t* lo, const bf16_t* hi) {
    const int n = threadIdx.x & 15, kg = (threadIdx.x & 63) >> 4;
    const bf16_t* base = (const bf16_t*)tile_row<SMALL>(lo, hi, n >= 8, ((8 * (n >> 2) + (n & 3)) * D + kg * 8) * 2);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int ks = 0; ks < Base::NKS; ++ks) this->ka[b][ks] = *(const bf16x8*)(base + 4 * b * D + ks * 32);
  }
  __device__ __forceinline__ void load_v(const bf16_t* lo, const bf16_t* hi) {
    const int n = threadIdx.x & 15, kg = (threadIdx.x & 63) >> 4;
    const bf16_t* base = (const bf16_t*)tile_row<SMALL>(lo, hi, kg >= 2, (8 * kg * D + n * Base::NV) * 2);
#pragma unroll
    for (int r = 0; r < 8; ++r) load_words<Base::NV / 2>(base + r * D, this->vw[r]);
  }
  __device__ __forceinline__ void clear_v(uint32_t seen) {          // bit r: the lane's key r
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int w = 0; w < Base::NV / 2; ++w) this->vw[r][w] = (seen >> r) & 1 ? this->vw[r][w] : 0u;
  }
  static __device__ __forceinline__ void load_q(const bf16_t* row, bool has, q_t (&qb)[NQ]) {
    const int kg = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int ks = 0; ks < NQ; ++ks) qb[ks] = has ? *(const bf16x8*)(row + ks * 32 + kg * 8) : bf16x8{};
  }
  // o += P V.  The factors are the upper 8 significant bits of the probabilities and, with `fine`, the next 8 too: the two are off by 2^-16 of the
  // probability at most (the upper ones alone by 2^-8; 64 requests' outputs 0.0017 and 0.0023 off, for 0.2 % of the time).  But an infinite
  // value times a second factor that is 0 or negative makes what the first one does not, so callers without finite results take the upper ones alone.
  static constexpr bool HAS_FINE = true;
  __device__ __forceinline__ void add(const float (&p)[8], dec_f32x4 (&o)[Base::NV], bool fine) const {
    const uint4 pk = make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7]));
    uint4 rk = make_uint4(0u, 0u, 0u, 0u);
    if (fine) {
      const uint32_t w[4] = {pk.x, pk.y, pk.z, pk.w};
      float rest[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) rest[j] = p[j] - __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
      rk = make_uint4(pack_bf16(rest[0], rest[1]), pack_bf16(rest[2], rest[3]), pack_bf16(rest[4], rest[5]), pack_bf16(rest[6], rest[7]));
    }
    const bf16x8 a = __builtin_bit_cast(bf16x8, pk), b = __builtin_bit_cast(bf16x8, rk);
#pragma unroll
    for (int w = 0; w < Base::NV / 2; ++w) {
#pragma unroll
      for (int up = 0; up < 2; ++up) {
        auto two = [&](int r) { return up ? upper_halves(this->vw[r][w], this->vw[r + 1][w]) : lower_halves(this->vw[r][w], this->vw[r + 1][w]); };
        const bf16x8 v = __builtin_bit_cast(bf16x8, make_uint4(two(0), two(2), two(4), two(6)));
        o[2 * w + up] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, v, o[2 * w + up], 0, 0, 0);
        if (fine) o[2 * w + up] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, v, o[2 * w + up], 0, 0, 0);
      }
    }
  }
};

// The same for float: v_mfma_f32_16x16x4_f32.  Contraction step (ks, e) of S^T has dim 16 ks + 4 kg + e in lane group kg, so that a lane
// reads 16 bytes; step r of a block's O = P V has key 4 kg + r there, which is where that key's probability is.
template <int D, bool SMALL> struct PagedTileF32 {
  static constexpr int NQ = D / 16, NV = D / 16;
  typedef float4 q_t;
  float4 ka[2][NQ];
  float vw[8][NV];
  __device__ __forceinline__ void load_k(const float* lo, const float* hi) {
    const int n = threadIdx.x & 15, kg = (threadIdx.x & 63) >> 4;
    const float* base = (const float*)tile_row<SMALL>(lo, hi, n >= 8, ((8 * (n >> 2) + (n & 3)) * D + kg * 4) * 4);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int ks = 0; ks < NQ; ++ks) ka[b][ks] = *(const float4*)(base + 4 * b * D + ks * 16);
  }
  __device__ __forceinline__ void load_v(const float* lo, const float* hi) {
    const int n = threadIdx.x & 15, kg = (threadIdx.x & 63) >> 4;
    const float* base = (const float*)tile_row<SMALL>(lo, hi, kg >= 2, (8 * kg * D + n * NV) * 4);
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int i = 0; i < NV; i += 2) *(float2*)&vw[r][i] = *(const float2*)(base + r * D + i);
  }
  __device__ __forceinline__ void clear_v(uint32_t seen) {
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int i = 0; i < NV; ++i) vw[r][i] = (seen >> r) & 1 ? vw[r][i] : 0.f;
  }
  static __device__ __forceinline__ void load_q(const float* row, bool has, q_t (&qb)[NQ]) {
    const int kg = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int ks = 0; ks < NQ; ++ks) qb[ks] = has ? *(const float4*)(row + ks * 16 + kg * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ __forceinline__ void logits(const q_t (&qb)[NQ], dec_f32x4 (&s)[2]) const {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      s[b] = dec_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < NQ; ++ks) {
        s[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka[b][ks].x, qb[ks].x, s[b], 0, 0, 0);
        s[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka[b][ks].y, qb[ks].y, s[b], 0, 0, 0);
        s[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka[b][ks].z, qb[ks].z, s[b], 0, 0, 0);
        s[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka[b][ks].w, qb[ks].w, s[b], 0, 0, 0);
      }
    }
  }
  static constexpr bool HAS_FINE = false;                  // 32-bit factors
  __device__ __forceinline__ void add(const float (&p)[8], dec_f32x4 (&o)[NV], bool) const {
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int i = 0; i < NV; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[r], vw[r][i], o[i], 0, 0, 0);
  }
};
template <typename T, int D, bool SMALL> struct PagedTileOf { typedef PagedTileBf16<D, SMALL> type; };
template <int D, bool SMALL> struct PagedTileOf<float, D, SMALL> { typedef PagedTileF32<D, SMALL> type; };

}  // namespace locret
