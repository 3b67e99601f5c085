// Internal interface of the paged entry points (paged_api.hip) to their kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace locret {

struct PagedDims {
  int h, h_kv, g, d;
  int bf16;
  int page_shift;       // log2 of the page size
  int n_pages;
  int max_pages;
  int window, n_sink;   // window 0: none; else less than the units of a row
  float scale;
};

// One step's bookkeeping (locret_paged_plan).
struct PagedPlan {
  int n_req, max_tokens, page_shift, n_pages, max_pages;
  const int32_t* lens;
  const int32_t* n_new;
  int32_t* lens_out;
  int32_t* table;
  int32_t* free_pages;
  const int32_t* n_free;
  int32_t* n_free_out;
  int32_t* cu_new;
  int32_t* slots;
  int32_t* positions;
};
constexpr int PAGED_MAX_REQS = 4096;
void launch_paged_plan(const PagedPlan& p, hipStream_t st);

struct PagedRows {
  int T;
  const void* q;
  const void* k;
  const void* v;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;      // strides in elements
  const int32_t* positions;
  const int32_t* slots;
  const double* freq;
  int rot, interleaved;
  float amplitude;
  const float* q_weight;
  const float* k_weight;
  float eps;
  void* q_out;
  void* K;
  void* V;
};
void launch_paged_append(const PagedDims& D, const PagedRows& a, hipStream_t st);

// Attention of T query tokens over pages.  cu NULL: token t is the last unit of request t (T = n_req).
struct PagedAttn {
  int n_req, T;
  const void* q;
  const void* K;
  const void* V;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* cu;
  void* out;
  float* lse;       // or NULL
  void* ws;
};
void launch_paged_decode(const PagedDims& D, const PagedAttn& a, hipStream_t st);
size_t paged_decode_workspace(const PagedDims& D, int max_reqs);
void launch_paged_prefill(const PagedDims& D, const PagedAttn& a, hipStream_t st);      // bf16
size_t paged_prefill_workspace(const PagedDims& D);
void launch_paged_prefill_f32(const PagedDims& D, const PagedAttn& a, hipStream_t st);
size_t paged_prefill_f32_workspace(const PagedDims& D);

// Workgroups of a launch over two grid dimensions: one dimension holds fewer than 2^32 threads.
inline dim3 paged_grid(int64_t n) { return n <= 1 << 20 ? dim3((unsigned)n) : dim3(1u << 20, (unsigned)((n + (1 << 20) - 1) >> 20)); }
__device__ __forceinline__ int paged_block() { return (int)(blockIdx.y * gridDim.x + blockIdx.x); }

// Data that a launch only reads, from places that are the same in a wavefront: through the scalar cache.
typedef const __attribute__((address_space(4))) int32_t* paged_const_i32;

// A length as the kernels take it.
__device__ __forceinline__ int paged_len(const int32_t* lens, int r, int max_pages, int page_shift) {
  return min(max(lens[r], 0), max_pages << page_shift);
}

// A position as the kernels compare it.  A chunk may be up to T tokens longer than its request: those in front of the first unit see nothing, at -1 as
// far below it, from where a window's first key is still a number of 32 bits.
__device__ __forceinline__ int paged_pos(int p) { return max(p, -1); }

__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Inclusive sums over the lanes of a wavefront: within rows of 16 lanes by shifts, then the last lane of each row on to the next ones.
__device__ __forceinline__ uint32_t wave_inclusive(uint32_t x) {
  x = add_sat(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));      // row_shr:1, 2, 4, 8
  x = add_sat(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = add_sat(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = add_sat(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = add_sat(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));      // row_bcast:15 into rows 1 and 3
  x = add_sat(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));      // row_bcast:31 into rows 2 and 3
  return x;
}
// Exclusive sums of N values over the workgroup's threads, and their totals; sums that pass 32 bits stay at 2^32 - 1.  part: N words a wavefront,
// free again after the next barrier.
template <int N> __device__ __forceinline__ void block_exclusive(const uint32_t (&x)[N], uint32_t (&before)[N], uint32_t (&total)[N], uint32_t* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
  uint32_t s[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    s[i] = wave_inclusive(x[i]);
    if (lane == 63) part[wave * N + i] = s[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) before[i] = total[i] = 0;
  for (int w = 0; w < nw; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t y = part[w * N + i];
      if (w < wave) before[i] = add_sat(before[i], y);
      total[i] = add_sat(total[i], y);
    }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t own = __shfl_up(s[i], 1, 64);                       // inclusive sum of the lane before
    before[i] = add_sat(before[i], lane ? own : 0u);
  }
}
__device__ __forceinline__ uint32_t block_exclusive(uint32_t x, uint32_t* part, uint32_t& total) {
  const uint32_t in[1] = {x};
  uint32_t before[1], all[1];
  block_exclusive<1>(in, before, all, part);
  total = all[0];
  return before[0];
}

// The last i in 0 .. n - 1 with first[i] <= x (first does not fall, first[0] <= x).
__device__ __forceinline__ int last_at_or_before(const int32_t* first, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// An entry of cu_new as the kernels take it.
__device__ __forceinline__ int paged_cu(const int32_t* cu, int r, int T) { return min(max(cu[r], 0), T); }

}  // namespace locret
