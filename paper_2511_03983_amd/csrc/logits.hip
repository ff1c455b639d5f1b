// Rules on the logits of a decoding step: penalties for repeated tokens, biases, grammar masks.
#include "nn.h"

namespace {

typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

template <int BF> __device__ __forceinline__ float load1(const void *p, int64_t i) {
  return BF ? __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16) : static_cast<const float *>(p)[i];
}
template <int BF> __device__ __forceinline__ f32x4v load4(const void *p, int64_t i) {
  if (!BF) return *reinterpret_cast<const f32x4v *>(static_cast<const float *>(p) + i);
  const u32x2v u = *reinterpret_cast<const u32x2v *>(static_cast<const uint16_t *>(p) + i);
  return f32x4v{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u)};
}

// What a row's rules say about a column, in one word of LDS: bit 0: in the history; then how often generated (COUNT bits); above that 1 + the column's last
// bias entry, or 0.  64 bits for lists that 32 cannot hold.
template <class Word> struct Fields { static constexpr int COUNT = sizeof(Word) == 4 ? 16 : 31, BIAS = COUNT + 1; };

// Bound by reading the logits and writing them in fp32, for few rows by the chain of loads: lengths, history, counts.  A workgroup of NT threads takes
// 16 NT columns of a row and has all their logits in flight while it counts in LDS what the row's history says about them (integers, so that any
// order of the atomics gives the same counts) and finds the last bias entry of each.  Four columns at a time where rows of input and output are
// aligned alike (from the first such column on: rows of an odd vocabulary start anywhere).
template <int BF, int NT, bool VEC, class Word>
__global__ __launch_bounds__(NT) void logits_kernel(const void *logits, int64_t ld, int V, twist_logit_rules R, float *out, int64_t ldo) {
  constexpr int COLS = 16 * NT, U = 4, H = 8, BIAS = Fields<Word>::BIAS;  // U, H: groups of four columns, and ids of the history, that a thread has in flight
  __shared__ __attribute__((aligned(16))) Word word[COLS + 4];
  __shared__ uint32_t allowed[COLS / 32 + 3];
  __shared__ float biases[NT];  // the first of the list
  const int t = blockIdx.y, tid = threadIdx.x;
  const int64_t in = t * ld;
  float *o = out + t * ldo;
  const int peel = VEC ? -(int)(reinterpret_cast<uintptr_t>(o) >> 2) & 3 : 0;
  const int base = blockIdx.x * COLS + peel, lo = blockIdx.x ? base : 0, hi = min(V, base + COLS), n = hi - lo;
  if (n <= 0) return;
  const int32_t *h = R.history + t * R.ld_history, *ids = R.bias_ids + t * R.ld_bias;
  const float *values = R.bias_values + t * R.ld_bias;
  unsigned ch[H];  // columns, counted from lo, that the first of the history are (what lies behind its length is not used)
#pragma unroll
  for (int u = 0; u < H; ++u) ch[u] = R.history && tid + u * NT < R.hist_cap ? (unsigned)h[tid + u * NT] - (unsigned)lo : ~0u;
  unsigned cb = R.bias_ids && tid < R.bias_cap ? (unsigned)ids[tid] - (unsigned)lo : ~0u;
  // the thread's columns: groups tid, tid + NT, ...; without alignment the columns lo + tid, lo + tid + NT, ...
  const int groups = hi > base ? (hi - base) / 4 : 0;
  f32x4v x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    x[u] = f32x4v{0.f, 0.f, 0.f, 0.f};
    if (VEC) {
      if (tid + u * NT < groups) x[u] = load4<BF>(logits, in + base + 4 * (tid + u * NT));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (lo + tid + (4 * u + e) * NT < hi) x[u][e] = load1<BF>(logits, in + lo + tid + (4 * u + e) * NT);
    }
  }
  const int nh = R.history ? min(R.n_history ? R.n_history[t] : R.hist_cap, R.hist_cap) : 0;
  const int nb = R.bias_ids ? min(R.n_bias ? R.n_bias[t] : R.bias_cap, R.bias_cap) : 0;
  const int np = nh > 0 && R.n_prompt ? R.n_prompt[t] : 0;
  const float rep = R.repetition ? R.repetition[t] : 1.f, freq = R.frequency ? R.frequency[t] : 0.f, pres = R.presence ? R.presence[t] : 0.f;
  const bool listed = nh > 0 || nb > 0;
  if (R.allowed)
    for (int i = tid; i <= (hi - 1) / 32 - lo / 32; i += NT) allowed[i] = R.allowed[t * R.ld_allowed + lo / 32 + i];
  if (listed) {
    const u32x4v zero = {0u, 0u, 0u, 0u};
    for (int i = tid; i < (int)((COLS + 4) * sizeof(Word) / 16); i += NT) reinterpret_cast<u32x4v *>(word)[i] = zero;
    const int shift = lo - base + 4;  // of a column counted from lo, in LDS
    __syncthreads();
    if (nb > 0) {
      if (tid < nb) biases[tid] = values[tid];
      for (int i = tid; i < nb; i += NT) {
        if (i != tid) cb = (unsigned)ids[i] - (unsigned)lo;
        if (cb < (unsigned)n) atomicMax(&word[cb + shift], (Word)(i + 1) << BIAS);
      }
      __syncthreads();
    }
    for (int i = tid; i < nh; i += H * NT) {
      if (i != tid) {
#pragma unroll
        for (int u = 0; u < H; ++u) ch[u] = i + u * NT < nh ? (unsigned)h[i + u * NT] - (unsigned)lo : ~0u;
      }
#pragma unroll
      for (int u = 0; u < H; ++u) {
        if (ch[u] >= (unsigned)n || i + u * NT >= nh) continue;
        if (i + u * NT < np) atomicOr(&word[ch[u] + shift], (Word)1);
        else atomicAdd(&word[ch[u] + shift], (Word)2);
      }
    }
  }
  __syncthreads();
  const float inv = 1.f / rep;  // (a rounding of 2^-24 more than the quotient, for a tenth of the instructions)
  auto ruled = [&](float v, Word w, bool may) {
    if (listed) {
      const uint32_t k = (uint32_t)(w & (((Word)1 << BIAS) - 1)), b = (uint32_t)(w >> BIAS);
      if (R.repetition) v *= k ? (v > 0.f ? inv : rep) : 1.f;
      v -= k > 1 ? fmaf(freq, (float)(k >> 1), pres) : 0.f;
      if (b) v += b <= NT ? biases[b - 1] : values[b - 1];
    }
    return may ? v : -INFINITY;
  };
  auto one = [&](float v, int c) { o[c] = ruled(v, word[c - base + 4], !R.allowed || (allowed[c / 32 - lo / 32] >> (c & 31) & 1)); };
  if (VEC) {
    if (tid < base - lo && lo + tid < hi) one(load1<BF>(logits, in + lo + tid), lo + tid);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int g = tid + u * NT, c = base + 4 * g;
      if (g >= groups) break;
      struct alignas(16) Four { Word w[4]; } four = {{0, 0, 0, 0}};
      if (listed) four = *reinterpret_cast<const Four *>(word + 4 * g + 4);
      uint32_t m = 15u;
      if (R.allowed) m = (uint32_t)(((uint64_t)allowed[c / 32 - lo / 32 + 1] << 32 | allowed[c / 32 - lo / 32]) >> (c & 31));
#pragma unroll
      for (int e = 0; e < 4; ++e) x[u][e] = ruled(x[u][e], four.w[e], m >> e & 1);
      *reinterpret_cast<f32x4v *>(o + c) = x[u];
    }
    const int c = base + 4 * groups + tid;
    if (tid < 4 && c >= base && c < hi) one(load1<BF>(logits, in + c), c);
  } else {
#pragma unroll
    for (int u = 0; u < 4 * U; ++u)
      if (lo + tid + u * NT < hi) one(x[u / 4][u % 4], lo + tid + u * NT);
  }
}

template <int BF>
void launch_logits(hipStream_t st, const void *logits, int64_t ld, int T, int V, const twist_logit_rules &r, float *out, int64_t ldo) {
  // whether a column that is 16-byte aligned in a row of the output is 4 elements aligned in the input's, whatever the row
  const int64_t es = BF ? 2 : 4, a = (int64_t)reinterpret_cast<uintptr_t>(logits), b = (int64_t)reinterpret_cast<uintptr_t>(out);
  const bool vec = a % es == 0 && b % 4 == 0 && (a / es - b / 4) % 4 == 0 && (ld - ldo) % 4 == 0;
  // every workgroup of a row reads its whole history.  512 threads (256, 1024): us, 1 x 50257 bf16 with 800 ids 5.7 (5.9, 6.3), 64 x 32000 with 2048 8.0 (10.2,
  // 8.6), 256 x 50257 fp32 with 4096 30.1 (32.7, 29.2); without any rule 3.5, 4.9, 17.
#define LOGITS(NT, VEC, WORD) \
  hipLaunchKernelGGL((logits_kernel<BF, NT, VEC, WORD>), dim3((unsigned)((V + 16 * NT - 1) / (16 * NT)), (unsigned)T), dim3(NT), 0, st, logits, ld, V, r, out, ldo)
  if (r.hist_cap < 1 << 16 && r.bias_cap < 1 << 15) { if (vec) LOGITS(512, true, uint32_t); else LOGITS(512, false, uint32_t); }
  else { if (vec) LOGITS(256, true, unsigned long long); else LOGITS(256, false, unsigned long long); }
#undef LOGITS
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
  if (V >= 1 << 30 || r.hist_cap >= 1 << 30 || r.bias_cap >= 1 << 30) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of 2^30 and more", who);
  if (ld < V || ldo < V) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows overlap", who);
  if (logits == static_cast<const void *>(out) && (ctx->d.dtype != TWIST_F32 || ld != ldo))
    TW_FAIL(ctx, TWIST_EINVAL, "%s: only fp32 logits can be changed in place", who);
  if (r.history && (r.hist_cap < 0 || r.ld_history < r.hist_cap)) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of the history overlap", who);
  if (r.bias_ids && !r.bias_values) TW_FAIL(ctx, TWIST_EINVAL, "%s: biased tokens without their biases", who);
  if (r.bias_ids && (r.bias_cap < 0 || r.ld_bias < r.bias_cap)) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of biases overlap", who);
  if (r.allowed && r.ld_allowed < ((int64_t)V + 31) / 32) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of the mask do not cover the vocabulary", who);
  if (ctx->d.dtype == TWIST_BF16) launch_logits<1>(ctx->stream, logits, ld, T, V, r, out, ldo);
  else launch_logits<0>(ctx->stream, logits, ld, T, V, r, out, ldo);
  TW_HIP(ctx, hipGetLastError());
  return TWIST_OK;
}
