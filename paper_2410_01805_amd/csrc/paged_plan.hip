// Block tables and slot maps of one serving step from the requests' lengths (locret_paged_plan).
//
// Whole numbers only.  With held = pages of a request's units, and over requests in their order
//   B_r = sum of held over the finished ones before r:   page p of finished request r goes to free_pages[n_free + B_r + p]
//   W_r = sum of the pages wanted before r:               page number held_r + i of request r is free_pages[F - 1 - W_r - i], F = all free
//   N_r = sum of new tokens before r:                     its token i is token N_r + i, at position len_r + i
// so everything follows from three prefix sums over at most 4096 requests, which one workgroup forms in registers and LDS
// (4 requests a thread).  Bound by latency: a step of 48 requests moves a kilobyte.  Up to PLAN_ONE tokens the same workgroup writes
// tables and slots too; more of them (prompts) are written by a second launch over all CUs, whose workgroups form the sums of W and N again
// from what the first one left (lens_out and cu_new give the lengths before the step), so that no workspace is needed
// and the lengths may be updated in place.
#include "paged.h"

namespace locret {

constexpr int PLAN_MAX_THREADS = 1024, PLAN_IPT = PAGED_MAX_REQS / PLAN_MAX_THREADS;
constexpr int PLAN_ONE = 4096;
constexpr int FILL_THREADS = 256, FILL_TOKENS = 4 * FILL_THREADS;

struct PlanSmem {
  int len[PAGED_MAX_REQS];          // units before the step (0 where the request is finished)
  int cu[PAGED_MAX_REQS + 1];       // N_r
  int want[PAGED_MAX_REQS + 1];     // W_r
  int64_t part[3][PLAN_MAX_THREADS / 64];
};

__device__ __forceinline__ int pages_of(int units, int shift) { return (int)(((int64_t)units + (1 << shift) - 1) >> shift); }

// Table entries of requests r0, r0 + r_step, ... (a wavefront each) and slots of the tokens [t0, t1), from the sums in LDS.
__device__ __forceinline__ void plan_fill(const PagedPlan& p, const PlanSmem& s, int n_all_free, int r0, int r_step, int t0, int t1) {
  const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 63;
  const int total = s.cu[p.n_req];
  for (int r = r0 + (tid >> 6); r < p.n_req; r += r_step) {
    const int held = pages_of(s.len[r], p.page_shift), n = s.want[r + 1] - s.want[r], top = n_all_free - 1 - s.want[r];
    for (int i = lane; i < n; i += 64) p.table[(int64_t)r * p.max_pages + held + i] = p.free_pages[top - i];
  }
  for (int t = t0 + tid; t < t1; t += nt) {
    int slot = -1, pos = 0;
    if (t < total) {
      int lo = 0, hi = p.n_req - 1;                    // the last request whose first token is at most t
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s.cu[mid] <= t) lo = mid; else hi = mid - 1;
      }
      pos = s.len[lo] + (t - s.cu[lo]);
      const int page = pos >> p.page_shift, i = page - pages_of(s.len[lo], p.page_shift);
      const int id = i < 0 ? p.table[(int64_t)lo * p.max_pages + page] : p.free_pages[n_all_free - 1 - s.want[lo] - i];
      if (id >= 0 && id < p.n_pages) slot = (id << p.page_shift) | (pos & ((1 << p.page_shift) - 1));      // (else the table or the list was not the pool's)
    }
    p.slots[t] = slot;
    p.positions[t] = pos;
  }
}

__global__ __launch_bounds__(PLAN_MAX_THREADS) void plan_kernel(PagedPlan p, int ipt, int fill) {
  __shared__ PlanSmem s;
  const int tid = threadIdx.x, nt = blockDim.x;
  const int most = p.max_pages << p.page_shift;
  int len[PLAN_IPT], add[PLAN_IPT];                    // add: tokens asked for, -1 finished
  int64_t back = 0, want = 0, tok = 0;
#pragma unroll
  for (int u = 0; u < PLAN_IPT; ++u) {
    const int r = tid * ipt + u;
    len[u] = add[u] = 0;
    if (u < ipt && r < p.n_req) {
      len[u] = min(max(p.lens[r], 0), most);
      add[u] = p.n_new[r];
      if (add[u] < 0) { add[u] = -1; back += pages_of(len[u], p.page_shift); }
      else if (add[u] > most - len[u]) add[u] = 0;
      if (add[u] > 0) {
        want += pages_of(len[u] + add[u], p.page_shift) - pages_of(len[u], p.page_shift);
        tok += add[u];
      }
    }
  }
  const int n_free = min(max(p.n_free[0], 0), p.n_pages);
  int64_t all_back, all_want, all_tok;
  int64_t b = block_exclusive(back, s.part[0], all_back);
  int64_t w = block_exclusive(want, s.part[1], all_want);
  int64_t n = block_exclusive(tok, s.part[2], all_tok);
  const int n_all_free = (int)(n_free + all_back < p.n_pages ? n_free + all_back : p.n_pages);
  // what fits, a prefix of the requests: both sums only grow
  int64_t w_in = 0, n_in = 0;                          // of the served ones of this thread
  bool fits = true;
#pragma unroll
  for (int u = 0; u < PLAN_IPT; ++u) {
    const int r = tid * ipt + u;
    if (u < ipt && r < p.n_req) {
      const int held = pages_of(len[u], p.page_shift);
      if (add[u] < 0) {
        const int32_t* row = p.table + (int64_t)r * p.max_pages;
        for (int i = 0; i < held; ++i)
          if (n_free + b + i < p.n_pages) p.free_pages[n_free + b + i] = row[i];
        b += held;
        len[u] = 0;
      }
      if (add[u] > 0) {
        const int pages = pages_of(len[u] + add[u], p.page_shift) - held;
        fits = fits && w + w_in + pages <= n_all_free && n + n_in + add[u] <= p.max_tokens;
        if (!fits) add[u] = 0;
        else { w_in += pages; n_in += add[u]; }
      }
    }
  }
  // Sums over the served ones.  A thread behind the first request that did not fit has served nothing, and its own sums lie
  // above the limits already, so the sums of all served requests are those of the last thread that served any.
  __syncthreads();                                     // part[] is free again, free_pages is complete for this workgroup
  int64_t sum_w, sum_n;
  const int64_t w0 = block_exclusive(w_in, s.part[0], sum_w), n0 = block_exclusive(n_in, s.part[1], sum_n);
  int cw = (int)w0, cn = (int)n0;
#pragma unroll
  for (int u = 0; u < PLAN_IPT; ++u) {
    const int r = tid * ipt + u;
    if (u < ipt && r < p.n_req) {
      s.len[r] = len[u];
      s.cu[r] = cn;
      s.want[r] = cw;
      p.cu_new[r] = cn;
      if (add[u] > 0) {
        cw += pages_of(len[u] + add[u], p.page_shift) - pages_of(len[u], p.page_shift);
        cn += add[u];
      }
      p.lens_out[r] = len[u] + max(add[u], 0);
    }
  }
  if (tid == 0) {
    s.cu[p.n_req] = (int)sum_n;
    s.want[p.n_req] = (int)sum_w;
    p.cu_new[p.n_req] = (int)sum_n;
    p.n_free_out[0] = n_all_free - (int)sum_w;
  }
  if (!fill) return;
  __syncthreads();
  plan_fill(p, s, n_all_free, 0, nt >> 6, 0, p.max_tokens);
}

// Tables and slots of a long step: workgroup b takes a share of the tokens and every gridDim.x-th four requests.
__global__ __launch_bounds__(FILL_THREADS) void plan_fill_kernel(PagedPlan p) {
  __shared__ PlanSmem s;
  const int tid = threadIdx.x;
  const int ipt = (p.n_req + FILL_THREADS - 1) / FILL_THREADS;
  int64_t want = 0, all;
  for (int u = 0; u < ipt; ++u) {
    const int r = tid * ipt + u;
    if (r < p.n_req) {
      const int c0 = p.cu_new[r], c1 = p.cu_new[r + 1], after = p.lens_out[r];
      s.len[r] = after - (c1 - c0);
      s.cu[r] = c0;
      const int pages = pages_of(after, p.page_shift) - pages_of(after - (c1 - c0), p.page_shift);
      s.want[r] = pages;
      want += pages;
      if (r == p.n_req - 1) s.cu[p.n_req] = c1;
    }
  }
  int64_t before = block_exclusive(want, s.part[0], all);
  for (int u = 0; u < ipt; ++u) {
    const int r = tid * ipt + u;
    if (r < p.n_req) { const int pages = s.want[r]; s.want[r] = (int)before; before += pages; }
  }
  if (tid == 0) s.want[p.n_req] = (int)all;
  __syncthreads();
  const int n_all_free = p.n_free_out[0] + (int)all;
  const int t0 = blockIdx.x * FILL_TOKENS, left = p.max_tokens - t0;
  plan_fill(p, s, n_all_free, blockIdx.x * (FILL_THREADS / 64), gridDim.x * (FILL_THREADS / 64), t0, t0 + min(left, FILL_TOKENS));
}

void launch_paged_plan(const PagedPlan& p, hipStream_t st) {
  const bool one = p.max_tokens <= PLAN_ONE || p.n_req == 0;
  const int threads = p.n_req <= 256 ? 256 : PLAN_MAX_THREADS;
  const int ipt = p.n_req > 0 ? (p.n_req + threads - 1) / threads : 1;
  plan_kernel<<<1, threads, 0, st>>>(p, ipt, one ? 1 : 0);
  if (!one) plan_fill_kernel<<<(unsigned)(((int64_t)p.max_tokens + FILL_TOKENS - 1) / FILL_TOKENS), FILL_THREADS, 0, st>>>(p);
}

}  // namespace locret
