// Rules on the logits of a decoding step: penalties for repeated tokens, biases, grammar masks.
#include "nn.h"

namespace {

constexpr int kT = 256;
constexpr int kCols = 4096;  // columns of a workgroup

// A workgroup per row and block of kCols columns.  It counts what the row's history says about its own columns in LDS (integer atomics: any
// order gives the same counts), finds the last bias entry of each, and then passes once over the logits.
template <int BF>
__global__ __launch_bounds__(kT) void logits_kernel(const void *logits, int64_t ld, int V, twist_logit_rules R, float *out, int64_t ldo) {
  __shared__ uint32_t cnt[kCols];   // bit 0: in the history; above it: how often generated
  __shared__ int32_t last[kCols];   // 1 + the last bias entry, or 0
  const int t = blockIdx.y, c0 = blockIdx.x * kCols, n = min(kCols, V - c0);
  for (int i = threadIdx.x; i < n; i += kT) { cnt[i] = 0; last[i] = 0; }
  __syncthreads();
  if (R.history) {
    const int nh = R.n_history ? min(R.n_history[t], R.hist_cap) : R.hist_cap, np = R.n_prompt ? R.n_prompt[t] : 0;
    for (int i = threadIdx.x; i < nh; i += kT) {
      const unsigned c = (unsigned)R.history[t * R.ld_history + i] - (unsigned)c0;
      if (c < (unsigned)n) {
        if (i < np) atomicOr(&cnt[c], 1u);
        else atomicAdd(&cnt[c], 2u);
      }
    }
  }
  if (R.bias_ids) {
    const int nb = R.n_bias ? min(R.n_bias[t], R.bias_cap) : R.bias_cap;
    for (int i = threadIdx.x; i < nb; i += kT) {
      const unsigned c = (unsigned)R.bias_ids[t * R.ld_bias + i] - (unsigned)c0;
      if (c < (unsigned)n) atomicMax(&last[c], i + 1);
    }
  }
  __syncthreads();
  const float rep = R.repetition ? R.repetition[t] : 1.f, freq = R.frequency ? R.frequency[t] : 0.f, pres = R.presence ? R.presence[t] : 0.f;
  for (int i = threadIdx.x; i < n; i += kT) {
    const int c = c0 + i;
    float x = BF ? __uint_as_float((uint32_t) static_cast<const uint16_t *>(logits)[t * ld + c] << 16) : static_cast<const float *>(logits)[t * ld + c];
    const uint32_t k = cnt[i];
    if (k) {
      if (R.repetition) x = x > 0.f ? x / rep : x * rep;
      if (k > 1) x = x - freq * (float)(k >> 1) - pres;
    }
    if (last[i]) x += R.bias_values[t * R.ld_bias + last[i] - 1];
    if (R.allowed && !(R.allowed[t * R.ld_allowed + (c >> 5)] >> (c & 31) & 1)) x = -INFINITY;
    out[t * ldo + c] = x;
  }
}

}  // namespace

extern "C" twist_status twist_logits_raw(twist_ctx *ctx, const void *logits, int64_t ld, int32_t T, const twist_logit_rules *rules, float *out, int64_t ldo) {
  const char *who = "twist_logits_raw";
  if (!ctx || !logits || !rules || !out) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  const int V = ctx->d.vocab;
  if (V < 1) TW_FAIL(ctx, TWIST_ESHAPE, "%s: needs a vocabulary", who);
  if (T < 1) TW_FAIL(ctx, TWIST_EINVAL, "%s: empty input", who);
  if (T > 65535) TW_FAIL(ctx, TWIST_ESHAPE, "%s: %d rows are too many for one call", who, T);
  const twist_logit_rules &r = *rules;
  if (ld < V || ldo < V) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows overlap", who);
  if (logits == static_cast<const void *>(out) && (ctx->d.dtype != TWIST_F32 || ld != ldo))
    TW_FAIL(ctx, TWIST_EINVAL, "%s: only fp32 logits can be changed in place", who);
  if (r.history && (r.hist_cap < 0 || r.ld_history < r.hist_cap)) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of the history overlap", who);
  if (r.bias_ids && !r.bias_values) TW_FAIL(ctx, TWIST_EINVAL, "%s: biased tokens without their biases", who);
  if (r.bias_ids && (r.bias_cap < 0 || r.ld_bias < r.bias_cap)) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of biases overlap", who);
  if (r.allowed && r.ld_allowed < ((int64_t)V + 31) / 32) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of the mask do not cover the vocabulary", who);
  const dim3 grid((unsigned)((V + kCols - 1) / kCols), (unsigned)T);
  if (ctx->d.dtype == TWIST_BF16) hipLaunchKernelGGL((logits_kernel<1>), grid, dim3(kT), 0, ctx->stream, logits, ld, V, r, out, ldo);
  else hipLaunchKernelGGL((logits_kernel<0>), grid, dim3(kT), 0, ctx->stream, logits, ld, V, r, out, ldo);
  TW_HIP(ctx, hipGetLastError());
  return TWIST_OK;
}
