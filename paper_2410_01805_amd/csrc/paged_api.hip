// Host side of the paged entry points of include/locret.h: argument checks and launches.  No state is kept between calls.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/locret.h"
#include "paged.h"

using namespace locret;

static_assert(PAGED_MAX_REQS == LOCRET_PAGED_MAX_REQS, "one limit");

namespace {

inline bool misaligned(const void* p, uintptr_t to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

int validate(const locret_paged_config* c, PagedDims* D) {
  if (!c) return LOCRET_EINVAL;
  if (c->dtype != LOCRET_F32 && c->dtype != LOCRET_BF16) return LOCRET_EINVAL;
  if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_pages < 1 || c->max_reqs < 1 || c->max_pages < 1 || c->window < 0 || c->n_sink < 0)
    return LOCRET_EINVAL;
  if (!(c->softmax_scale >= 0.f) || !isfinite(c->softmax_scale)) return LOCRET_EINVAL;
  if (c->n_q_heads % c->n_kv_heads != 0 || c->n_q_heads > 1024 || c->n_q_heads / c->n_kv_heads > 128) return LOCRET_ESHAPE;
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128) return LOCRET_ESHAPE;
  int shift = 0;
  for (int s = 4; s <= 8; ++s) if (c->page_size == 1 << s) shift = s;
  if (!shift || c->max_reqs > PAGED_MAX_REQS) return LOCRET_ESHAPE;
  if (((int64_t)c->n_pages << shift) > INT32_MAX || ((int64_t)c->max_pages << shift) > 1 << 30) return LOCRET_ESHAPE;
  if (((int64_t)c->max_reqs * c->max_pages << shift) > (int64_t)1 << 37) return LOCRET_ESHAPE;     // units of work are counted in 32 bits
  D->h = c->n_q_heads;
  D->h_kv = c->n_kv_heads;
  D->g = D->h / D->h_kv;
  D->d = c->head_dim;
  D->bf16 = c->dtype == LOCRET_BF16;
  D->page_shift = shift;
  D->n_pages = c->n_pages;
  D->max_pages = c->max_pages;
  // a window that reaches over a whole row hides nothing; the others are below 2^30, so that position - window stays in 32 bits
  D->window = (int64_t)c->window >= (int64_t)c->max_pages << shift ? 0 : c->window;
  D->n_sink = c->n_sink;
  D->scale = c->softmax_scale > 0.f ? c->softmax_scale : 1.0f / sqrtf((float)c->head_dim);
  return LOCRET_OK;
}

size_t workspace_bytes(const PagedDims& D, int max_reqs) {
  const size_t a = paged_decode_workspace(D, max_reqs), b = D.bf16 ? paged_prefill_workspace(D) : paged_prefill_f32_workspace(D);
  return a > b ? a : b;
}

int launched() { return hipGetLastError() == hipSuccess ? LOCRET_OK : LOCRET_EHIP; }

int attention(const locret_paged_config* cfg, const PagedAttn& a, size_t bytes, bool prefill, hipStream_t st) {
  PagedDims D;
  const int rc = validate(cfg, &D);
  if (rc != LOCRET_OK) return rc;
  if (a.n_req < 0 || a.T < 0) return LOCRET_EINVAL;
  // (launches are counted in 32 bits, the float prefill's rows of a request too)
  if (a.n_req > cfg->max_reqs || (int64_t)a.T * D.h > (int64_t)1 << (D.bf16 ? 34 : 31)) return LOCRET_ESHAPE;
  if (a.n_req == 0 || a.T == 0) return LOCRET_OK;
  if (!a.q || !a.K || !a.V || !a.table || !a.lens || (prefill && !a.cu) || !a.out || !a.ws) return LOCRET_EINVAL;
  if (misaligned(a.q) || misaligned(a.K) || misaligned(a.V) || misaligned(a.out) || misaligned(a.ws, 256) || misaligned(a.table, 4) ||
      misaligned(a.lens, 4) || misaligned(a.cu, 4) || misaligned(a.lse, 4))
    return LOCRET_EALIGN;
  if (bytes < workspace_bytes(D, cfg->max_reqs)) return LOCRET_ENOMEM;
  if (prefill && D.bf16) launch_paged_prefill(D, a, st);
  else if (prefill) launch_paged_prefill_f32(D, a, st);
  else launch_paged_decode(D, a, st);
  return launched();
}

}  // namespace

extern "C" {

size_t locret_paged_workspace_bytes(const locret_paged_config* cfg) {
  PagedDims D;
  return validate(cfg, &D) == LOCRET_OK ? workspace_bytes(D, cfg->max_reqs) : 0;
}

int locret_paged_plan(const locret_paged_config* cfg, int32_t n_req, const int32_t* lens, const int32_t* n_new, int32_t* lens_out,
                      int32_t* block_table, int32_t* free_pages, const int32_t* n_free, int32_t* n_free_out, int32_t max_tokens,
                      int32_t* cu_new, int32_t* slots, int32_t* positions, void* stream) {
  PagedDims D;
  const int rc = validate(cfg, &D);
  if (rc != LOCRET_OK) return rc;
  if (n_req < 0 || max_tokens < 0 || !free_pages || !n_free || !n_free_out || !cu_new) return LOCRET_EINVAL;
  if (n_req > 0 && (!lens || !n_new || !lens_out || !block_table)) return LOCRET_EINVAL;
  if (max_tokens > 0 && (!slots || !positions)) return LOCRET_EINVAL;
  if (n_req > cfg->max_reqs) return LOCRET_ESHAPE;
  const void* p[] = {lens, n_new, lens_out, block_table, free_pages, n_free, n_free_out, cu_new, slots, positions};
  for (const void* x : p) if (misaligned(x, 4)) return LOCRET_EALIGN;
  const PagedPlan plan = {n_req, max_tokens, D.page_shift, D.n_pages, D.max_pages, lens, n_new, lens_out, block_table, free_pages, n_free,
                          n_free_out, cu_new, slots, positions};
  launch_paged_plan(plan, (hipStream_t)stream);
  return launched();
}

int locret_rope_frequencies(const locret_rope_config* c, double* freq, float* amplitude) {
  if (!c || !freq || !amplitude) return LOCRET_EINVAL;
  if (c->scaling < LOCRET_ROPE_PLAIN || c->scaling > LOCRET_ROPE_FACTORS) return LOCRET_EINVAL;
  if (c->rotary_dim < 2 || c->rotary_dim > 4096 || c->rotary_dim % 2) return LOCRET_ESHAPE;
  if (!(c->theta > 1.0) || !isfinite(c->theta)) return LOCRET_EINVAL;
  const bool by_length = c->scaling >= LOCRET_ROPE_BANDS, bounds = c->scaling == LOCRET_ROPE_BANDS || c->scaling == LOCRET_ROPE_RAMP;
  if (c->scaling != LOCRET_ROPE_PLAIN && (!(c->factor > 0.0) || !isfinite(c->factor))) return LOCRET_EINVAL;
  if (by_length && (!(c->original > 1.0) || !isfinite(c->original))) return LOCRET_EINVAL;
  if (bounds && !(c->low > 0.0 && c->high > c->low && isfinite(c->high))) return LOCRET_EINVAL;
  const int n = c->rotary_dim / 2;
  if (c->scaling == LOCRET_ROPE_FACTORS) {
    if (!c->factors) return LOCRET_EINVAL;
    for (int i = 0; i < n; ++i) if (!(c->factors[i] > 0.0) || !isfinite(c->factors[i])) return LOCRET_EINVAL;
  }
  const double two_pi = 6.283185307179586476925;
  double first = 0, last = 0;          // RAMP: the pairs between which frequencies are mixed
  if (c->scaling == LOCRET_ROPE_RAMP) {
    // pair i turns r = original theta^(-2i/rotary_dim) / 2 pi times over the first context
    auto pair_of = [&](double r) { return c->rotary_dim * log(c->original / (r * two_pi)) / (2.0 * log(c->theta)); };
    first = fmax(floor(pair_of(c->high)), 0.0);
    last = fmin(ceil(pair_of(c->low)), (double)(c->rotary_dim - 1));
    if (last <= first) last = first + 0.001;      // a step
  }
  for (int i = 0; i < n; ++i) {
    const double f = pow(c->theta, -2.0 * i / c->rotary_dim);
    double keep = 1.0;                 // weight of f itself against f / factor
    if (c->scaling == LOCRET_ROPE_LINEAR) keep = 0.0;
    if (c->scaling == LOCRET_ROPE_BANDS) keep = fmin(1.0, fmax(0.0, (c->original * f / two_pi - c->low) / (c->high - c->low)));
    if (c->scaling == LOCRET_ROPE_RAMP) keep = 1.0 - fmin(1.0, fmax(0.0, (i - first) / (last - first)));
    freq[i] = c->scaling == LOCRET_ROPE_FACTORS ? f / c->factors[i] : keep == 1.0 ? f : keep * f + (1.0 - keep) * f / c->factor;
  }
  *amplitude = 1.f;
  if (c->scaling == LOCRET_ROPE_RAMP && c->factor > 1.0) *amplitude = (float)(0.1 * log(c->factor) + 1.0);
  if (c->scaling == LOCRET_ROPE_FACTORS && c->factor > 1.0) *amplitude = (float)sqrt(1.0 + log(c->factor) / log(c->original));
  return LOCRET_OK;
}

int locret_paged_append(const locret_paged_config* cfg, int32_t T, const void* q, const void* k, const void* v, const int64_t* strides,
                        const int32_t* positions, const int32_t* slots, const double* freq, int32_t rotary_dim,
                        int32_t interleaved, float amplitude, const float* q_weight, const float* k_weight, float eps,
                        void* q_out, void* K, void* V, void* stream) {
  PagedDims D;
  const int rc = validate(cfg, &D);
  if (rc != LOCRET_OK) return rc;
  if (T < 0 || (interleaved != 0 && interleaved != 1) || !isfinite(amplitude) || !(eps >= 0.f) || !isfinite(eps)) return LOCRET_EINVAL;
  if (rotary_dim < 0 || rotary_dim > D.d || rotary_dim % 16) return LOCRET_ESHAPE;
  if (T == 0) return LOCRET_OK;
  if ((!q && !k) || (q && !q_out) || !k != !v || (k && (!K || !V || !slots)) || (rotary_dim && (!freq || !positions))) return LOCRET_EINVAL;
  const int64_t d = D.d, dense[6] = {D.h * d, d, D.h_kv * d, d, D.h_kv * d, d};
  const int64_t* s = strides ? strides : dense;
  const int vec = D.bf16 ? 8 : 4;
  // a stride that leads nowhere, of one token or one head, may be anything
  auto used = [&](int i) { return i & 1 ? (i < 2 ? D.h : D.h_kv) > 1 : T > 1; };
  for (int i = 0; i < 6; ++i) {
    if (!(i < 2 ? q : k) || !used(i)) continue;
    if (s[i] < 0) return LOCRET_EINVAL;
    if (s[i] % vec) return LOCRET_EALIGN;
  }
  for (int i = 0; i < 2; ++i) if (q && q_out == q && used(i) && s[i] != dense[i]) return LOCRET_EINVAL;
  const void* p[] = {q, k, v, q_out, K, V, q_weight, k_weight};
  for (const void* x : p) if (misaligned(x)) return LOCRET_EALIGN;
  if (misaligned(positions, 4) || misaligned(slots, 4) || misaligned(freq, 8)) return LOCRET_EALIGN;
  const PagedRows a = {T, q, k, v, s[0], s[1], s[2], s[3], s[4], s[5], positions, slots, freq, rotary_dim, interleaved, amplitude, q_weight,
                       k_weight, eps, q_out, K, V};
  launch_paged_append(D, a, (hipStream_t)stream);
  return launched();
}

int locret_paged_decode(const locret_paged_config* cfg, int32_t n_req, const void* q, const void* K, const void* V,
                        const int32_t* block_table, const int32_t* lens, void* out, float* lse, void* workspace,
                        size_t workspace_bytes, void* stream) {
  const PagedAttn a = {n_req, n_req, q, K, V, block_table, lens, nullptr, out, lse, workspace};
  return attention(cfg, a, workspace_bytes, false, (hipStream_t)stream);
}

int locret_paged_prefill(const locret_paged_config* cfg, int32_t n_req, int32_t T, const void* q, const void* K, const void* V,
                         const int32_t* block_table, const int32_t* lens, const int32_t* cu_new, void* out, float* lse,
                         void* workspace, size_t workspace_bytes, void* stream) {
  const PagedAttn a = {n_req, T, q, K, V, block_table, lens, cu_new, out, lse, workspace};
  return attention(cfg, a, workspace_bytes, true, (hipStream_t)stream);
}

}  // extern "C"
