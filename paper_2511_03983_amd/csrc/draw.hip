// What is taken from a row of logits: a token drawn from it, or its k largest.  A row's columns have one order, larger logits first and equal ones by column; everything here is a
// beginning of it.
#include "nn.h"

namespace {

constexpr int kT = 256;
constexpr int kTop = 1024;  // the longest list

template <int BF> __device__ __forceinline__ float load1(const void *p, int64_t i) {
  const float v = BF ? __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16) : static_cast<const float *>(p)[i];
  return v == v ? v + 0.f : -INFINITY;  // no number: -infinity; -0 is 0
}

// Unsigned numbers in the order of the logits, and of a row's columns: the place in 32 bits, the column (turned over) below it.
__device__ __forceinline__ uint32_t value_key(float v) {
  const uint32_t b = __float_as_uint(v);
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ uint64_t place(float v, int c) { return (uint64_t)value_key(v) << 32 | (0xffffffffu - (uint32_t)c); }

template <class T> __device__ __forceinline__ T block_add(T v, T *sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}
template <class T> __device__ __forceinline__ T block_most(T v, T *sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (T)__shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return max(max(sh[0], sh[1]), max(sh[2], sh[3]));
}

// The last place of the shortest beginning whose columns' amounts add up to `target` (at least 1, at most the whole row's), by halving what is left of the places: 64 passes.
template <int BF, class F> __device__ uint64_t reach(const void *x, int64_t row, int V, uint64_t target, unsigned long long *sh, F amount) {
  uint64_t lo = 0, hi = ~0ull;  // the beginning down to lo is long enough, the one down to hi + 1 is not
  while (lo < hi) {
    const uint64_t mid = hi - (hi - lo) / 2;
    unsigned long long n = 0;
    for (int c = threadIdx.x; c < V; c += kT) {
      const float v = load1<BF>(x, row + c);
      if (place(v, c) >= mid) n += amount(v);
    }
    if (block_add(n, sh) >= target) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// A row a workgroup.  Sums of probabilities are whole multiples of 2^-bits of the largest, formed in 64 bits from exponentials in 64: any order gives the same, and a column's share of them
// is exact to far less than the random number's last place.
template <int BF>
__global__ __launch_bounds__(kT) void draw_kernel(const void *x, int64_t ld, int V, int bits, const float *uniform, twist_draw_rules R, int32_t *tokens, float *logprobs, int32_t *kept) {
  __shared__ unsigned long long sh[4];
  const int t = blockIdx.x;
  const int64_t row = t * ld;
  uint64_t first = 0;
  unsigned long long n = 0;
  for (int c = threadIdx.x; c < V; c += kT) {
    const float v = load1<BF>(x, row + c);
    const uint64_t p = place(v, c);
    first = p > first ? p : first;
    n += v > -INFINITY;
  }
  first = block_most((unsigned long long)first, sh);
  n = block_add(n, sh);
  const float top = key_value((uint32_t)(first >> 32)), temp = R.temperature ? R.temperature[t] : 1.f;
  if (n == 0 || !(temp > 0.f)) {
    if (threadIdx.x == 0) {
      tokens[t] = n ? (int32_t)(0xffffffffu - (uint32_t)first) : -1;
      if (logprobs) logprobs[t] = n ? 0.f : -INFINITY;
      if (kept) kept[t] = n ? 1 : 0;
    }
    return;
  }
  const double scale = ldexp(1.0, bits);
  auto exponent = [&](float v) { return v == top ? 0.0 : fmax(((double)v - (double)top) / (double)temp, -1e5); };  // (also where that is no number)
  auto mass = [&](float v) -> unsigned long long { return v > -INFINITY ? (unsigned long long)(exp(exponent(v)) * scale + 0.5) : 0; };
  auto one = [](float v) -> unsigned long long { return v > -INFINITY; };
  auto sum_from = [&](uint64_t from) {
    unsigned long long m = 0;
    for (int c = threadIdx.x; c < V; c += kT) {
      const float v = load1<BF>(x, row + c);
      if (place(v, c) >= from) m += mass(v);
    }
    return block_add(m, sh);
  };
  // the last place that each rule keeps
  uint64_t last = 0;
  if (R.top_k && R.top_k[t] > 0 && (unsigned)R.top_k[t] < n) last = reach<BF>(x, row, V, R.top_k[t], sh, one);
  unsigned long long total = sum_from(last);
  if (R.top_p && R.top_p[t] < 1.f) {
    const double share = ceil((double)R.top_p[t] * (double)total);
    const uint64_t p = reach<BF>(x, row, V, share >= 1.0 ? min((unsigned long long)share, total) : 1, sh, mass);
    last = p > last ? p : last;
  }
  if (R.min_p && R.min_p[t] > 0.f) {
    const double least = min((double)R.min_p[t], 1.0);
    uint32_t lo = (uint32_t)(last >> 32), hi = (uint32_t)(first >> 32);  // of the values that may be kept, the smallest that is probable enough
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo) / 2;
      if (exp(exponent(key_value(mid))) >= least) hi = mid;
      else lo = mid + 1;
    }
    if (lo > (uint32_t)(last >> 32)) last = (uint64_t)lo << 32;
  }
  total = sum_from(last);
  n = 0;
  for (int c = threadIdx.x; c < V; c += kT) {
    const float v = load1<BF>(x, row + c);
    n += v > -INFINITY && place(v, c) >= last;
  }
  n = block_add(n, sh);
  const float u = uniform[t];
  const unsigned long long at = u > 0.f ? min((unsigned long long)((double)u * (double)total), total - 1) : 0;
  const uint64_t p = reach<BF>(x, row, V, at + 1, sh, mass);
  if (threadIdx.x == 0) {
    tokens[t] = (int32_t)(0xffffffffu - (uint32_t)p);
    if (logprobs) logprobs[t] = (float)(exponent(key_value((uint32_t)(p >> 32))) - log((double)total / scale));
    if (kept) kept[t] = (int32_t)n;
  }
}

template <int BF>
__global__ __launch_bounds__(kT) void top_kernel(const void *x, int64_t ld, int V, int k, float inv_temp, int32_t *ids, float *values, int64_t ldk, float *rest) {
  __shared__ unsigned long long sh[4], list[kTop];
  __shared__ float shf[4];
  __shared__ int count;
  const int64_t row = blockIdx.x * ld, out = blockIdx.x * ldk;
  const int n = min(k, V);
  const uint64_t last = n < V ? reach<BF>(x, row, V, n, sh, [](float) -> unsigned long long { return 1; }) : 0;
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  float m = -INFINITY;
  for (int c = threadIdx.x; c < V; c += kT) {
    const float v = load1<BF>(x, row + c);
    const uint64_t p = place(v, c);
    if (p >= last) list[atomicAdd(&count, 1)] = p;
    else m = fmaxf(m, v);
  }
  m = block_most(m, shf);
  for (int i = threadIdx.x; i < k; i += kT) {
    int at = i;
    if (i < n) {
      at = 0;
      for (int j = 0; j < n; ++j) at += list[j] > list[i];
    }
    ids[out + at] = i < n ? (int32_t)(0xffffffffu - (uint32_t)list[i]) : -1;
    values[out + at] = i < n ? key_value((uint32_t)(list[i] >> 32)) : -INFINITY;
  }
  if (!rest) return;
  float s = 0.f;
  for (int c = threadIdx.x; c < V; c += kT) {
    const float v = load1<BF>(x, row + c);
    if (place(v, c) < last && v > -INFINITY) s += v == m ? 1.f : __expf((v - m) * inv_temp);
  }
  s = block_add(s, shf);
  if (threadIdx.x == 0) rest[blockIdx.x] = m > -INFINITY ? m * inv_temp + logf(s) : -INFINITY;
}

twist_status check_rows(twist_ctx *ctx, const char *who, int64_t ld, int T) {
  const int V = ctx->d.vocab;
  if (V < 1) TW_FAIL(ctx, TWIST_ESHAPE, "%s: needs a vocabulary", who);
  if (T < 1) TW_FAIL(ctx, TWIST_EINVAL, "%s: empty input", who);
  if (T >= 1 << 22) TW_FAIL(ctx, TWIST_ESHAPE, "%s: %d rows are too many for one call", who, T);
  if (V >= 1 << 20) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of 2^20 and more", who);
  if (ld < V) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows overlap", who);
  return TWIST_OK;
}

}  // namespace

extern "C" twist_status twist_draw_raw(twist_ctx *ctx, const void *logits, int64_t ld, int32_t logits_f32, int32_t T, const float *uniform, const twist_draw_rules *rules,
                                       int32_t *tokens, float *logprobs, int32_t *kept) {
  const char *who = "twist_draw_raw";
  if (!ctx || !logits || !uniform || !tokens) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  TW_TRY(check_rows(ctx, who, ld, T));
  const int V = ctx->d.vocab;
  int bits = 51;  // no row's sum reaches 2^63
  while (V > (int64_t)1 << (62 - bits)) --bits;
  const twist_draw_rules r = rules ? *rules : twist_draw_rules{};
  if (ctx->d.dtype == TWIST_BF16 && !logits_f32) hipLaunchKernelGGL((draw_kernel<1>), dim3(T), dim3(kT), 0, ctx->stream, logits, ld, V, bits, uniform, r, tokens, logprobs, kept);
  else hipLaunchKernelGGL((draw_kernel<0>), dim3(T), dim3(kT), 0, ctx->stream, logits, ld, V, bits, uniform, r, tokens, logprobs, kept);
  TW_HIP(ctx, hipGetLastError());
  return TWIST_OK;
}

extern "C" twist_status twist_top_logits_raw(twist_ctx *ctx, const void *logits, int64_t ld, int32_t logits_f32, int32_t T, int32_t k, float temperature, int32_t *ids,
                                             float *values, int64_t ldk, float *rest) {
  const char *who = "twist_top_logits_raw";
  if (!ctx || !logits || !ids || !values) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  TW_TRY(check_rows(ctx, who, ld, T));
  if (k < 1 || k > kTop) TW_FAIL(ctx, TWIST_ESHAPE, "%s: lists of %d entries (1 to %d)", who, k, kTop);
  if (ldk < k) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of the lists overlap", who);
  if (!(temperature > 0.f && temperature < INFINITY)) TW_FAIL(ctx, TWIST_EINVAL, "%s: the temperature must be above 0 and finite", who);
  const float inv = 1.f / temperature;
  if (ctx->d.dtype == TWIST_BF16 && !logits_f32) hipLaunchKernelGGL((top_kernel<1>), dim3(T), dim3(kT), 0, ctx->stream, logits, ld, ctx->d.vocab, k, inv, ids, values, ldk, rest);
  else hipLaunchKernelGGL((top_kernel<0>), dim3(T), dim3(kT), 0, ctx->stream, logits, ld, ctx->d.vocab, k, inv, ids, values, ldk, rest);
  TW_HIP(ctx, hipGetLastError());
  return TWIST_OK;
}
