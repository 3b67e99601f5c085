// Queries, keys and values of new tokens on their way into attention and the pages (locret_paged_append): RMS norm per
// head, rotation, queries out, keys and values to their slots, in one pass over the data.
//
//   y = x / sqrt(mean x^2 + eps) * weight;   (a, b) -> (a c - b s, b c + a s),  c, s = amplitude * cos, sin(position * f_i)
//
// Bound by HBM: every element is read once and written once, the sums of a row stay in the lanes that hold it.  A lane holds two
// 16-byte chunks of a row, the partners of a rotation where the pairs are (i, i + rot/2), neighbours otherwise, so that
// neither the rotation nor an update in place needs another lane's data.  A workgroup has one token (8192 tokens of 32 query and 8 KV heads of
// 128 dims: 40.2 us, 5.0 TB/s, what a large copy reaches; with 2, 4, 8 tokens 41.9, 43.7, 44.7), whose angles it forms once, in LDS, for all
// heads: the turns position * f / 2 pi in 64 bits, of which only the fraction goes on in 32 (a product in 32 bits is
// rounded by up to 2^-24 of it, at position 2^20 by 2^-4 radians; the fraction is rounded by 2^-25 turns, 2^-22 radians).
#include "device_util.h"
#include "paged.h"

namespace locret {

constexpr int APPEND_THREADS = 256;

template <typename T, int D, bool IL>
__global__ __launch_bounds__(APPEND_THREADS) void paged_append_kernel(PagedRows a, int h, int h_kv, int page_shift, int n_pages) {
  constexpr int VEC = Vec16<T>::N;
  constexpr int LPR = D / (2 * VEC);                         // lanes that hold a row
  constexpr int LPRP = LPR <= 2 ? 2 : LPR <= 4 ? 4 : LPR <= 8 ? 8 : 16;
  constexpr int RPP = APPEND_THREADS / LPRP;                 // rows the workgroup takes at a time
  typedef Vec16<T> V16;
  typedef decltype(V16().raw) raw_t;
  __shared__ float2 turn[D / 2];                             // [rot / 2]: amplitude * (cos, sin)
  const int tid = threadIdx.x, half = a.rot >> 1, t = paged_block();
  if (t >= a.T) return;
  if (tid < half) {
    const double turns = (double)a.positions[t] * a.freq[tid] * 0.15915494309189533577;
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    turn[tid] = make_float2(a.amplitude * c, a.amplitude * s);
  }
  __syncthreads();
  const int sub = tid % LPRP, HR = half / VEC;
  const bool act = sub < LPR;
  const int lane_c = act ? sub : 0;
  // the lane's two chunks
  const int c0 = !IL && lane_c < HR ? lane_c : 2 * lane_c, c1 = !IL && lane_c < HR ? lane_c + HR : 2 * lane_c + 1;
  const int nq = a.q ? h : 0, nk = a.k ? h_kv : 0, R = nq + 2 * nk;
  const int slot = a.k ? a.slots[t] : -1;
  const bool has = slot >= 0 && (slot >> page_shift) < n_pages;
  for (int rr = tid / LPRP; rr < R; rr += RPP) {
    const bool isq = rr < nq, isk = !isq && rr < nq + nk;
    const int head = isq ? rr : isk ? rr - nq : rr - nq - nk;
    const T* src = isq ? (const T*)a.q + t * a.q_tok + head * a.q_head
                       : isk ? (const T*)a.k + t * a.k_tok + head * a.k_head : (const T*)a.v + t * a.v_tok + head * a.v_head;
    T* dst;
    if (isq) {
      dst = (T*)a.q_out + ((int64_t)t * h + head) * D;
    } else {
      const int64_t at = (((int64_t)(slot >> page_shift) * h_kv + head) << page_shift) + (slot & ((1 << page_shift) - 1));
      dst = has ? (T*)(isk ? a.K : a.V) + at * D : nullptr;
    }
    V16 x, y;
    x.raw = *(const raw_t*)(src + c0 * VEC);
    y.raw = *(const raw_t*)(src + c1 * VEC);
    if (isq || isk) {
      float u[VEC], w[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) { u[e] = x.get(e); w[e] = y.get(e); }
      const float* weight = isq ? a.q_weight : a.k_weight;
      if (weight) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) ss = fmaf(u[e], u[e], fmaf(w[e], w[e], ss));
        if (!act) ss = 0.f;
#pragma unroll
        for (int by = 1; by < LPRP; by <<= 1) ss += __shfl_xor(ss, by, 64);
        const float inv = 1.f / sqrtf(ss * (1.f / D) + a.eps);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          u[e] = u[e] * inv * weight[c0 * VEC + e];
          w[e] = w[e] * inv * weight[c1 * VEC + e];
        }
      }
      const float2* cs = turn;
      if constexpr (IL) {
        if (c0 * VEC < a.rot) {
#pragma unroll
          for (int e = 0; e < VEC; e += 2) {
            const float2 p = cs[(c0 * VEC + e) >> 1], r = cs[(c1 * VEC + e) >> 1];
            const float u0 = u[e], w0 = w[e];
            u[e] = u0 * p.x - u[e + 1] * p.y;
            u[e + 1] = u[e + 1] * p.x + u0 * p.y;
            w[e] = w0 * r.x - w[e + 1] * r.y;
            w[e + 1] = w[e + 1] * r.x + w0 * r.y;
          }
        }
      } else if (lane_c < HR) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float2 p = cs[c0 * VEC + e];
          const float u0 = u[e];
          u[e] = u0 * p.x - w[e] * p.y;
          w[e] = w[e] * p.x + u0 * p.y;
        }
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) { x.set(e, u[e]); y.set(e, w[e]); }
    }
    if (act && dst) {
      *(raw_t*)(dst + c0 * VEC) = x.raw;
      *(raw_t*)(dst + c1 * VEC) = y.raw;
    }
  }
}

template <typename T, int D>
static void append_d(const PagedDims& Dm, const PagedRows& a, hipStream_t st) {
  if (a.interleaved) paged_append_kernel<T, D, true><<<paged_grid(a.T), APPEND_THREADS, 0, st>>>(a, Dm.h, Dm.h_kv, Dm.page_shift, Dm.n_pages);
  else paged_append_kernel<T, D, false><<<paged_grid(a.T), APPEND_THREADS, 0, st>>>(a, Dm.h, Dm.h_kv, Dm.page_shift, Dm.n_pages);
}

void launch_paged_append(const PagedDims& D, const PagedRows& a, hipStream_t st) {
#define LOCRET_APPEND(T)                        \
  switch (D.d) {                                \
    case 32: append_d<T, 32>(D, a, st); break;  \
    case 64: append_d<T, 64>(D, a, st); break;  \
    case 96: append_d<T, 96>(D, a, st); break;  \
    default: append_d<T, 128>(D, a, st); break; \
  }
  if (D.bf16) { LOCRET_APPEND(bf16_t) } else { LOCRET_APPEND(float) }
#undef LOCRET_APPEND
}

}  // namespace locret
