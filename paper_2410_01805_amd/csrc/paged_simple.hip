// Attention over pages in its simplest form: one wavefront per query token and head.
//   S_j = scale q . k_j over the visible keys j, out = sum_j exp(S_j - M) v_j / sum_j exp(S_j - M), lse = M + ln(sum)
// A step takes 64 keys, a lane each: its dot product, the running maximum and sum of the softmax, then all lanes go over the 64 values, a dim each.
#include "device_util.h"
#include "paged.h"

namespace locret {

template <typename T, int D>
__global__ __launch_bounds__(64) void paged_attn_simple_kernel(PagedAttn a, PagedDims Dm) {
  constexpr int NO = (D + 63) / 64;
  __shared__ float qs[D];
  __shared__ float ps[64];
  __shared__ int64_t at[64];
  const int t = blockIdx.x, j = blockIdx.y, m = j / Dm.g, lane = threadIdx.x;
  const int page = 1 << Dm.page_shift;
  int r = t, pos;
  if (a.cu) {
    for (r = 0; r < a.n_req; ++r)
      if (t >= paged_cu(a.cu, r, a.T) && t < paged_cu(a.cu, r + 1, a.T)) break;
    if (r == a.n_req) return;
    pos = paged_len(a.lens, r, Dm.max_pages, Dm.page_shift) - (paged_cu(a.cu, r + 1, a.T) - t);
  } else {
    pos = paged_len(a.lens, r, Dm.max_pages, Dm.page_shift) - 1;
  }
  const int64_t row = (int64_t)t * Dm.h + j;
  const float c = Dm.scale * 1.4426950408889634f;
  for (int e = lane; e < D; e += 64) qs[e] = Elem<T>::ld((const T*)a.q + row * D + e) * c;
  __syncthreads();
  float M = -INFINITY, L = 0.f, o[NO];
  for (int i = 0; i < NO; ++i) o[i] = 0.f;
  const int w0 = Dm.window ? max(0, pos - Dm.window + 1) : 0, ns = min(Dm.n_sink, w0);
  for (int base = 0; base < ns + (pos + 1 - w0); base += 64) {
    const int i = base + lane, key = i < ns ? i : i - ns + w0;
    const int id = key <= pos ? a.table[(int64_t)r * Dm.max_pages + (key >> Dm.page_shift)] : -1;
    float s = -INFINITY;
    at[lane] = -1;
    if (id >= 0 && id < Dm.n_pages) {
      at[lane] = ((((int64_t)id * Dm.h_kv + m) << Dm.page_shift) + (key & (page - 1))) * D;
      s = 0.f;
      for (int e = 0; e < D; ++e) s = fmaf(qs[e], Elem<T>::ld((const T*)a.K + at[lane] + e), s);
    }
    float mx = s;
    for (int by = 32; by; by >>= 1) mx = fmaxf(mx, __shfl_xor(mx, by, 64));
    mx = fmaxf(mx, M);
    const float ref = mx == -INFINITY ? 0.f : mx, alpha = exp2f(M - ref);
    const float p = exp2f(s - ref);
    float sum = p;
    for (int by = 32; by; by >>= 1) sum += __shfl_xor(sum, by, 64);
    ps[lane] = p;
    __syncthreads();
    L = L * alpha + sum;
    M = mx;
    for (int i2 = 0; i2 < NO; ++i2) o[i2] *= alpha;
    for (int k = 0; k < 64; ++k) {
      if (at[k] < 0) continue;
      for (int i2 = 0; i2 < NO; ++i2)
        if (i2 * 64 + lane < D) o[i2] = fmaf(ps[k], Elem<T>::ld((const T*)a.V + at[k] + i2 * 64 + lane), o[i2]);
    }
    __syncthreads();
  }
  const bool none = M == -INFINITY && L == 0.f;
  for (int i = 0; i < NO; ++i)
    if (i * 64 + lane < D) Elem<T>::st((T*)a.out + row * D + i * 64 + lane, none ? 0.f : o[i] / L);
  if (a.lse && lane == 0) a.lse[row] = none ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

void launch_paged_attn_simple(const PagedDims& D, const PagedAttn& a, hipStream_t st) {
  const dim3 grid((unsigned)a.T, (unsigned)D.h);
#define LOCRET_SIMPLE(T)                                                             \
  switch (D.d) {                                                                     \
    case 32: paged_attn_simple_kernel<T, 32><<<grid, 64, 0, st>>>(a, D); break;      \
    case 64: paged_attn_simple_kernel<T, 64><<<grid, 64, 0, st>>>(a, D); break;      \
    case 96: paged_attn_simple_kernel<T, 96><<<grid, 64, 0, st>>>(a, D); break;      \
    default: paged_attn_simple_kernel<T, 128><<<grid, 64, 0, st>>>(a, D); break;     \
  }
  if (D.bf16) { LOCRET_SIMPLE(bf16_t) } else { LOCRET_SIMPLE(float) }
#undef LOCRET_SIMPLE
}

}  // namespace locret
