// The loss of a student's logits against a teacher's top logits and the targets, with its gradient.
#include "nn.h"

namespace {

constexpr int kT = 256;
constexpr int kTop = 1024;  // the longest list

template <int BF> __device__ __forceinline__ float load1(const void *p, int64_t i) {
  return BF ? __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16) : static_cast<const float *>(p)[i];
}
template <int BF> __device__ __forceinline__ void store1(void *p, int64_t i, float v) {
  if (BF) static_cast<__bf16 *>(p)[i] = (__bf16)v;  // round to nearest even
  else static_cast<float *>(p)[i] = v;
}

template <class T> __device__ __forceinline__ T block_add(T v, T *sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}
__device__ __forceinline__ float block_max(float v, float *sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3]));
}

// Natural logarithm of a / (a + b), near 1 as exact as far from it.
__device__ __forceinline__ double log_share(double a, double b) { return b < a ? -log1p(b / a) : log(a / (a + b)); }

// A row a workgroup.  The row's tokens are the teacher's (the set) and the others, whose share of the distribution is formed from themselves and not as what the set leaves: it may be
// next to nothing, or all but everything.  With tau the temperature, p and q over the set and over the others together (P, Q of them), the gradient of
// KL(q || p) is (p_i - q_i) / tau in the set and p_i (P - Q) / P / tau outside it.  WORDS: 32 tokens each, of the table of which are in the set.
template <int BF, int WORDS>
__global__ __launch_bounds__(kT) void distill_kernel(const void *x, int64_t ld, const int32_t *targets, int V, twist_teacher te, void *grad, int64_t ldg, int64_t pad, float inv_T,
                                                     float *rowloss) {
  __shared__ uint32_t in_set[WORDS];
  __shared__ int32_t id[kTop];
  __shared__ float logit[kTop];
  __shared__ double weight[kTop];
  __shared__ double shd[4];
  __shared__ float shf[4];
  __shared__ int twice;
  const int t = blockIdx.x, tid = threadIdx.x, k = te.k;
  const int64_t row = t * ld, out = t * ldg;
  const float tau = te.temperature, inv_tau = 1.f / tau;
  for (int i = tid; i < (V + 31) / 32; i += kT) in_set[i] = 0;
  if (tid == 0) twice = 0;
  __syncthreads();
  float mt = te.rest ? te.rest[t] : -INFINITY;
  const float rest = mt;
  float mine = -INFINITY, other = -INFINITY;  // largest logits of the set and of the others
  for (int j = tid; j < k; j += kT) {
    const int c = te.ids[t * te.ld + j];
    const bool on = (unsigned)c < (unsigned)V;
    id[j] = on ? c : -1;
    if (!on) continue;
    if (atomicOr(&in_set[c / 32], 1u << (c & 31)) >> (c & 31) & 1) twice = 1;
    logit[j] = load1<BF>(x, row + c);
    mine = fmaxf(mine, logit[j]);
    mt = fmaxf(mt, te.values[t * te.ld + j] * inv_tau);
  }
  mt = block_max(mt, shf);
  const int tgt = te.weight < 1.f ? targets[t] : -1;
  const bool taught = te.weight > 0.f && mt > -INFINITY, aimed = (unsigned)tgt < (unsigned)V;
  if (!taught && !aimed) {
    for (int c = tid; c < pad; c += kT) store1<BF>(grad, out + c, 0.f);
    if (tid == 0) rowloss[t] = 0.f;
    return;
  }
  // the teacher's weights against its largest; of a token that is named twice the first entry takes the others'
  for (int j = tid; j < k; j += kT)
    if (id[j] >= 0) weight[j] = taught ? exp((double)te.values[t * te.ld + j] / tau - (double)mt) : 0.0;
  const double rest_weight = taught && rest > -INFINITY ? exp((double)rest - (double)mt) : 0.0;
  __syncthreads();
  if (twice) {
    double sum[kTop / kT];
    bool first[kTop / kT];
    for (int j = tid, u = 0; j < k; j += kT, ++u) {
      sum[u] = 0.0;
      first[u] = id[j] >= 0;
      for (int i = 0; i < k; ++i)
        if (id[i] == id[j]) {
          sum[u] += weight[i];
          first[u] = first[u] && i >= j;
        }
    }
    __syncthreads();
    for (int j = tid, u = 0; j < k; j += kT, ++u) {
      if (!first[u]) id[j] = -1;
      else weight[j] = sum[u];
    }
  }
  auto outside = [&](int c) { return !(in_set[c / 32] >> (c & 31) & 1); };
  for (int c = tid; c < V; c += kT) other = fmaxf(other, outside(c) ? load1<BF>(x, row + c) : -INFINITY);
  mine = block_max(mine, shf);
  other = block_max(other, shf);
  const float m = fmaxf(mine, other);
  float s1 = 0.f, st = 0.f;
  for (int c = tid; c < V; c += kT)
    if (outside(c) && other > -INFINITY) {
      const float d = load1<BF>(x, row + c) - other;
      s1 += __expf(d);
      st += __expf(d * inv_tau);
    }
  // sums over the others, brought to the row's largest, and over the set
  const double down = other > -INFINITY ? (double)other - m : 0.0;
  const double others1 = block_add((double)s1, shd) * exp(down), others = block_add((double)st, shd), others_m = others * exp(down / tau);
  double set1 = 0.0, set = 0.0, qs = 0.0;
  for (int j = tid; j < k; j += kT)
    if (id[j] >= 0) {
      const double d = (double)logit[j] - m;
      set1 += exp(d);
      set += exp(d / tau);
      qs += weight[j];
    }
  set1 = block_add(set1, shd);
  set = block_add(set, shd);
  qs = block_add(qs, shd);
  const double z1 = others1 + set1, z = others_m + set, zq = qs + rest_weight;
  const double log_z = log(z), log_zq = log(zq);
  const double log_others = others_m > 0.0 ? log_share(others_m, set) : down / tau + (others > 0.0 ? log(others) : -INFINITY) - log_z;
  double kl = 0.0;
  if (taught)
    for (int j = tid; j < k; j += kT)
      if (id[j] >= 0 && weight[j] != 0.0) kl += weight[j] / zq * ((log(weight[j]) - log_zq) - (((double)logit[j] - m) / tau - log_z));
  kl = block_add(kl, shd);
  const double Q = taught ? rest_weight / zq : 0.0, P = others_m / z;
  if (rest_weight != 0.0) kl += Q * (log_share(rest_weight, qs) - log_others);
  // the others' gradient is their share of each other times P - Q, which is what the set's probabilities differ by
  const double more = Q < 0.5 ? P - Q : qs / zq - set / z;
  const float a1 = aimed ? (float)((1.0 - (double)te.weight) / z1 * inv_T) : 0.f, at = taught && others > 0.0 ? (float)((double)te.weight * tau * more / others * inv_T) : 0.f;
  for (int c = tid; c < V; c += kT) {
    const float v = load1<BF>(x, row + c);
    float g = at != 0.f ? __expf((v - other) * inv_tau) * at : 0.f;
    if (aimed) g += __expf(v - m) * a1 - (c == tgt ? (1.f - te.weight) * inv_T : 0.f);
    if (c == tgt && tid == c % kT) rowloss[t] = (float)((double)te.weight * tau * tau * kl + (1.0 - (double)te.weight) * (log(z1) - ((double)v - m)));
    store1<BF>(grad, out + c, g);
  }
  for (int64_t c = V + tid; c < pad; c += kT) store1<BF>(grad, out + c, 0.f);
  if (!aimed && tid == 0) rowloss[t] = (float)((double)te.weight * tau * tau * kl);
  __syncthreads();  // (the set's gradients take the places of what was written above)
  for (int j = tid; j < k; j += kT)
    if (id[j] >= 0) {
      const double d = (double)logit[j] - m;
      double g = taught ? (double)te.weight * tau * (exp(d / tau) / z - weight[j] / zq) : 0.0;
      if (aimed) g += (1.0 - (double)te.weight) * (exp(d) / z1 - (id[j] == tgt ? 1.0 : 0.0));
      store1<BF>(grad, out + id[j], (float)(g * inv_T));
    }
}

}  // namespace

twist_status twist_check_teacher(twist_ctx *ctx, const char *who, const twist_teacher *te, int T, int V) {
  if (V < 1) TW_FAIL(ctx, TWIST_ESHAPE, "%s: needs a vocabulary", who);
  if (T < 1) TW_FAIL(ctx, TWIST_EINVAL, "%s: empty input", who);
  if (T >= 1 << 22) TW_FAIL(ctx, TWIST_ESHAPE, "%s: %d rows are too many for one call", who, T);
  if (V >= 1 << 20) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of 2^20 and more", who);
  if (!te->ids || !te->values) TW_FAIL(ctx, TWIST_EINVAL, "%s: the teacher's list is missing", who);
  if (te->k < 1 || te->k > kTop) TW_FAIL(ctx, TWIST_ESHAPE, "%s: lists of %d entries (1 to %d)", who, te->k, kTop);
  if (te->ld < te->k) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of the lists overlap", who);
  if (!(te->temperature > 0.f && te->temperature < INFINITY)) TW_FAIL(ctx, TWIST_EINVAL, "%s: the temperature must be above 0 and finite", who);
  if (!(te->weight >= 0.f && te->weight <= 1.f)) TW_FAIL(ctx, TWIST_EINVAL, "%s: the teacher's weight must be in 0 .. 1", who);
  return TWIST_OK;
}

twist_status twist_distill(twist_ctx *ctx, const char *who, int bf16, const void *logits, int64_t ld, const int32_t *targets, int T, int V, const twist_teacher *te, void *grad, int64_t ldg,
                           int64_t pad, float *rowloss, float *loss) {
  TW_TRY(twist_check_teacher(ctx, who, te, T, V));
  const float inv_T = 1.f / (float)T;
#define DISTILL(BF, WORDS) \
  hipLaunchKernelGGL((distill_kernel<BF, WORDS>), dim3(T), dim3(kT), 0, ctx->stream, logits, ld, targets, V, *te, grad, ldg, pad, inv_T, rowloss)
  if (V <= 1 << 16) { if (bf16) DISTILL(1, 1 << 11); else DISTILL(0, 1 << 11); }
  else { if (bf16) DISTILL(1, 1 << 15); else DISTILL(0, 1 << 15); }
#undef DISTILL
  return twist_mean(ctx, rowloss, T, inv_T, loss);
}

extern "C" twist_status twist_distill_raw(twist_ctx *ctx, const void *logits, int64_t ld, const int32_t *targets, int32_t T, const twist_teacher *teacher, void *grad, int64_t ldg,
                                          float *rowloss, float *loss) {
  const char *who = "twist_distill_raw";
  if (!ctx || !logits || !teacher || !grad || !rowloss || !loss) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  const int V = ctx->d.vocab;
  TW_TRY(twist_check_teacher(ctx, who, teacher, T, V));
  if (teacher->weight < 1.f && !targets) TW_FAIL(ctx, TWIST_EINVAL, "%s: targets are missing", who);
  if (ld < V || ldg < V) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows overlap", who);
  if (logits == grad && ld != ldg) TW_FAIL(ctx, TWIST_EINVAL, "%s: a gradient in the logits' place has their rows", who);
  return twist_distill(ctx, who, ctx->d.dtype == TWIST_BF16, logits, ld, targets, T, V, teacher, grad, ldg, V, rowloss, loss);
}
