// The loss of a student's logits against a teacher's top logits and the targets, with its gradient.
#include "nn.h"

namespace {

constexpr int kTop = 1024;  // the longest list
constexpr float kLog2e = 1.44269504f;

typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

// Sixteen bytes of a row, from any element on, as floats: eight of bf16, four of fp32.  (Rows of an odd vocabulary start anywhere; loads and stores need no alignment.)
template <int BF> struct Piece {
  static constexpr int N = BF ? 8 : 4, ES = BF ? 2 : 4;
  u32x4v u;
  __device__ __forceinline__ void load(const char *row, int v) { __builtin_memcpy(&u, row + (int64_t)v * 16, 16); }
  static __device__ __forceinline__ u32x4v none() {  // -infinity throughout
    const uint32_t n = BF ? 0xff80ff80u : 0xff800000u;
    return u32x4v{n, n, n, n};
  }
  __device__ __forceinline__ float operator[](int e) const {
    if (!BF) return __uint_as_float(u[e % 4]);
    return __uint_as_float(e % 2 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16);
  }
  __device__ __forceinline__ void clear(uint32_t bits) {  // -infinity where a bit is set
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (bits >> e & 1) {
        if (BF) u[e / 2] = e % 2 ? (u[e / 2] & 0xffffu) | 0xff800000u : (u[e / 2] & 0xffff0000u) | 0xff80u;
        else u[e % 4] = 0xff800000u;
      }
  }
};
template <int BF> __device__ __forceinline__ float load1(const char *row, int c) {
  return BF ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(row)[c] << 16) : reinterpret_cast<const float *>(row)[c];
}
template <int BF> __device__ __forceinline__ void store1(char *row, int64_t c, float v) {
  if (BF) reinterpret_cast<__bf16 *>(row)[c] = (__bf16)v;  // round to nearest even
  else reinterpret_cast<float *>(row)[c] = v;
}
template <int BF> __device__ __forceinline__ void store_piece(char *row, int v, const float *g) {
  u32x4v u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    if (BF) u[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{g[2 * i % Piece<BF>::N], g[(2 * i + 1) % Piece<BF>::N]}), b2));
    else u[i] = __float_as_uint(g[i]);
  }
  __builtin_memcpy(row + (int64_t)v * 16, &u, 16);
}

template <class T> __device__ __forceinline__ T wave_add(T v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// exp(x) in 32 bits: the exponent's rounding, which a large one would multiply, taken care of
__device__ __forceinline__ float exp_f32(double x) {
  const double y = x * 1.4426950408889634;
  if (y <= -200.0) return 0.f;
  const float h = (float)y;
  return __builtin_amdgcn_exp2f(h) * fmaf((float)(y - h), 0.69314718f, 1.f);
}

// Natural logarithm of a / (a + b), near 1 as exact as far from it.
__device__ __forceinline__ double log_share(double a, double b) { return b < a ? -log1p(b / a) : log(a / (a + b)); }

// A row a workgroup.  The row's tokens are the teacher's (the set) and the others, whose share of the distribution is formed from themselves and not as what the set leaves: it may be
// next to nothing, or all but everything.  With tau the temperature, p and q over the set and over the others together (P, Q of them), the gradient of
// KL(q || p) is (p_i - q_i) / tau in the set and p_i (P - Q) / P / tau outside it.
// Bound by memory: the row is read once and its gradient written once.  It stays in registers as it came (NV pieces of 16 bytes a thread; rows that NT threads cannot hold, NV = 0, are read
// three times), the set's columns as -infinity, so that they weigh nothing in the others' sums; their own gradients, a thread each and in 64 bits where they meet a logarithm, are stored over
// the others' behind a barrier.
template <int BF, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void distill_kernel(const char *logits, int64_t ld, const int32_t *targets, int V, twist_teacher te, char *grads, int64_t ldg, int64_t pad, float inv_T,
                                                     float *rowloss) {
  using P16 = Piece<BF>;
  constexpr int N = P16::N, NW = NT / 64, WORDS = NV ? NV * NT * N / 32 : 1 << 15;
  __shared__ uint32_t in_set[WORDS];  // a bit a column
  __shared__ int32_t id[kTop];
  __shared__ float logit[kTop];
  __shared__ double weight[kTop], part[kTop];  // the teacher's weights against its largest, and their exponents
  __shared__ float most[3][NW], sums[2][NW];
  __shared__ double set_sums[3][NW], kls[NW];
  __shared__ int twice;
  const int t = blockIdx.x, tid = threadIdx.x, k = te.k, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const char *row = logits + (int64_t)t * ld * P16::ES;
  char *out = grads + (int64_t)t * ldg * P16::ES;
  const double tau = te.temperature, inv_tau = 1.0 / tau;
  const int pieces = V / N, mine = pieces - 64 * wave;  // u NT >= mine: the wave's piece u lies beyond the row
  const int last = pieces * N + tid;                    // the row's last columns, fewer than a piece, a thread each
  P16 x[NV ? NV : 1];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    x[u].u = P16::none();
    if (u * NT + tid < pieces) x[u].load(row, u * NT + tid);
  }
  float xl = last < V ? load1<BF>(row, last) : -INFINITY;
  const int tgt = te.weight < 1.f ? targets[t] : -1;
  const bool aimed = (unsigned)tgt < (unsigned)V;
  const float rest = te.rest ? te.rest[t] : -INFINITY, aim = aimed ? load1<BF>(row, tgt) : 0.f;
  for (int i = tid; i < (V + 31) / 32; i += NT) in_set[i] = 0;
  if (tid == 0) twice = 0;
  __syncthreads();
  float top_t = rest, top_set = -INFINITY;  // largest of the teacher's, and of the student's in the set
  for (int j = tid; j < k; j += NT) {
    const int c = te.ids[t * te.ld + j];
    const bool on = (unsigned)c < (unsigned)V;
    id[j] = on ? c : -1;
    if (!on) continue;
    if (atomicOr(&in_set[c / 32], 1u << (c & 31)) >> (c & 31) & 1) twice = 1;
    logit[j] = load1<BF>(row, c);
    top_set = fmaxf(top_set, logit[j]);
    top_t = fmaxf(top_t, (float)(te.values[t * te.ld + j] * inv_tau));
  }
  top_t = wave_max(top_t);
  top_set = wave_max(top_set);
  if (lane == 0) { most[0][wave] = top_t; most[1][wave] = top_set; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) { top_t = fmaxf(top_t, most[0][w]); top_set = fmaxf(top_set, most[1][w]); }
  const bool taught = te.weight > 0.f && top_t > -INFINITY;
  if (!taught && !aimed) {
    const float zeros[N] = {};
    for (int v = tid; v < pieces; v += NT) store_piece<BF>(out, v, zeros);
    for (int64_t c = last; c < pad; c += NT) store1<BF>(out, c, 0.f);
    if (tid == 0) rowloss[t] = 0.f;
    return;
  }
  auto bits_of = [&](int v) {  // of a piece's columns in the set
    const uint32_t b = reinterpret_cast<const uint8_t *>(in_set)[N == 8 ? v : v / 2];
    return N == 8 ? b : b >> (v % 2 * 4) & 15u;
  };
  // f(piece, its number) for all of the thread's pieces of the row, those beyond it and the set's columns -infinity
  auto each = [&](auto f) {
    if (NV) {
      int at = tid;
      asm volatile("" : "+v"(at));  // (neither places nor what one pass makes of the pieces are kept for the next: registers)
#pragma unroll
      for (int u = 0; u < NV; ++u)
        if (u * NT < mine) {
          asm volatile("" : "+v"(x[u].u));
          f(x[u], u * NT + at);
        }
    } else {
      for (int v = tid; v < pieces; v += NT) {
        P16 y;
        y.load(row, v);
        y.clear(bits_of(v));
        f(y, v);
      }
    }
  };
#pragma unroll
  for (int u = 0; u < NV; ++u)
    if (u * NT < mine) {
      const uint32_t b = bits_of(u * NT + tid);
      if (b) x[u].clear(b);
    }
  if (last < V && in_set[last / 32] >> (last & 31) & 1) xl = -INFINITY;
  float other = xl;
  each([&](const P16 &y, int) {
#pragma unroll
    for (int e = 0; e < N; ++e) other = fmaxf(other, y[e]);
  });
  other = wave_max(other);
  if (lane == 0) most[2][wave] = other;
  // the teacher's weights against its largest; of a token that is named twice the first entry takes the others'
  for (int j = tid; j < k; j += NT)
    if (id[j] >= 0) {
      part[j] = te.values[t * te.ld + j] * inv_tau - top_t;
      weight[j] = taught ? exp(part[j]) : 0.0;
    }
  const double rest_weight = taught && rest > -INFINITY ? exp((double)rest - (double)top_t) : 0.0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) other = fmaxf(other, most[2][w]);
  if (twice) {
    constexpr int M = (kTop + NT - 1) / NT;
    double sum[M];
    bool first[M];
#pragma unroll
    for (int u = 0; u < M; ++u) {
      const int j = u * NT + tid;
      sum[u] = 0.0;
      first[u] = j < k && id[j] >= 0;
      if (first[u])
        for (int i = 0; i < k; ++i)
          if (id[i] == id[j]) {
            sum[u] += weight[i];
            first[u] = first[u] && i >= j;
          }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < M; ++u) {
      const int j = u * NT + tid;
      if (j < k && !first[u]) id[j] = -1;
      else if (j < k && sum[u] != weight[j]) {
        weight[j] = sum[u];
        part[j] = log(sum[u]);
      }
    }
  }
  const float ref = other > -INFINITY ? other : 0.f, m = fmaxf(top_set, other);
  // sums over the others against their largest, and over the set against the row's
  const float c1 = kLog2e, ct = (float)(kLog2e * inv_tau);
  float s1 = __builtin_amdgcn_exp2f((xl - ref) * c1), st = __builtin_amdgcn_exp2f((xl - ref) * ct);
  each([&](const P16 &y, int) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float d = y[e] - ref;
      if (aimed) s1 += __builtin_amdgcn_exp2f(d * c1);
      if (taught) st += __builtin_amdgcn_exp2f(d * ct);
    }
  });
  double set1 = 0.0, set = 0.0, qs = 0.0;
  for (int j = tid; j < k; j += NT)
    if (id[j] >= 0) {
      const double d = (double)logit[j] - m;
      if (aimed) set1 += exp_f32(d);
      if (taught) set += exp(d * inv_tau);
      qs += weight[j];
    }
  s1 = wave_add(s1);
  st = wave_add(st);
  if (64 * wave < k) { set1 = wave_add(set1); set = wave_add(set); qs = wave_add(qs); }
  if (lane == 0) {
    sums[0][wave] = s1; sums[1][wave] = st;
    set_sums[0][wave] = set1; set_sums[1][wave] = set; set_sums[2][wave] = qs;
  }
  __syncthreads();
  double others1 = 0.0, others = 0.0;
  set1 = set = qs = 0.0;
#pragma unroll 4
  for (int w = 0; w < NW; ++w) {
    others1 += sums[0][w]; others += sums[1][w];
    set1 += set_sums[0][w]; set += set_sums[1][w]; qs += set_sums[2][w];
  }
  const double down = other > -INFINITY ? (double)other - m : 0.0;
  const float down1 = __expf((float)down), others_m = (float)others * __builtin_amdgcn_exp2f((float)down * ct);
  const float z1 = fmaf((float)others1, down1, (float)set1), z = others_m + (float)set, zq = (float)(qs + rest_weight);
  const float iz1 = 1.f / z1, iz = 1.f / z, izq = 1.f / zq, Q = taught ? (float)rest_weight * izq : 0.f, P = others_m * iz;
  // the others' gradient is their share of each other times P - Q, which is what the set's probabilities differ by
  const float more = Q < 0.5f ? P - Q : (float)qs * izq - (float)set * iz;
  const float w1 = (1.f - te.weight) * inv_T, wt = te.weight * te.temperature * inv_T;
  const float a1 = aimed ? w1 * down1 * iz1 : 0.f, at = taught && others > 0.0 ? wt * more / (float)others : 0.f;
  each([&](const P16 &y, int v) {
    float g[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float d = y[e] - ref;
      g[e] = 0.f;
      if (aimed) g[e] = __builtin_amdgcn_exp2f(d * c1) * a1;
      if (taught) g[e] = fmaf(__builtin_amdgcn_exp2f(d * ct), at, g[e]);
    }
    if (v < pieces) store_piece<BF>(out, v, g);
  });
  for (int64_t c = last; c < pad; c += NT)
    store1<BF>(out, c, c == last && c < V ? (aimed ? __builtin_amdgcn_exp2f((xl - ref) * c1) * a1 : 0.f) + (taught ? __builtin_amdgcn_exp2f((xl - ref) * ct) * at : 0.f) : 0.f);
  // the row's loss, in 64 bits
  const double whole = others * exp(down * inv_tau) + set;
  double kl = 0.0;
  if (taught && 64 * wave < k) {
    const double shift = log(whole) - log(qs + rest_weight);
    for (int j = tid; j < k; j += NT)
      if (id[j] >= 0 && weight[j] != 0.0) kl += weight[j] * (part[j] - ((double)logit[j] - m) * inv_tau + shift);
    kl = wave_add(kl);
  }
  if (lane == 0) kls[wave] = kl;
  __syncthreads();  // (the set's gradients take the places of what was written above, and so does the target's)
  for (int j = tid; j < k; j += NT)
    if (id[j] >= 0) {
      const double d = (double)logit[j] - m;
      float g = taught ? wt * (exp_f32(d * inv_tau) * iz - (float)weight[j] * izq) : 0.f;
      if (aimed) g += w1 * (exp_f32(d) * iz1 - (id[j] == tgt ? 1.f : 0.f));
      store1<BF>(out, id[j], g);
    }
  if (tid == 0) {
    double loss = 0.0;
    if (aimed) {
      loss = (1.0 - (double)te.weight) * (log(others1 * exp(down) + set1) - ((double)aim - m));
      if (!(in_set[tgt / 32] >> (tgt & 31) & 1)) {
        const float d = aim - ref;
        store1<BF>(out, tgt, (__builtin_amdgcn_exp2f(d * c1) * a1 - w1) + (taught ? __builtin_amdgcn_exp2f(d * ct) * at : 0.f));
      }
    }
    if (taught) {
      kl = 0.0;
      for (int w = 0; w < NW; ++w) kl += kls[w];
      kl /= qs + rest_weight;
      if (rest_weight != 0.0) {
        const double rm = others * exp(down * inv_tau), log_others = rm > 0.0 ? log_share(rm, set) : down * inv_tau + (others > 0.0 ? log(others) : -INFINITY) - log(whole);
        kl += rest_weight / (qs + rest_weight) * (log_share(rest_weight, qs) - log_others);
      }
      loss += (double)te.weight * tau * tau * kl;
    }
    rowloss[t] = (float)loss;
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
  const char *x = static_cast<const char *>(logits);
  char *g = static_cast<char *>(grad);
#define DISTILL(BF, NT, NV) hipLaunchKernelGGL((distill_kernel<BF, NT, NV>), dim3(T), dim3(NT), 0, ctx->stream, x, ld, targets, V, *te, g, ldg, pad, inv_T, rowloss)
  if (bf16) {
    if (V <= 4 * 8 * 256) DISTILL(1, 256, 4);
    else if (V <= 16 * 8 * 256) DISTILL(1, 256, 16);
    else if (V <= 16 * 8 * 512) DISTILL(1, 512, 16);
    else DISTILL(1, 1024, 0);
  } else {
    if (V <= 4 * 4 * 256) DISTILL(0, 256, 4);
    else if (V <= 16 * 4 * 256) DISTILL(0, 256, 16);
    else if (V <= 16 * 4 * 512) DISTILL(0, 512, 16);
    else if (V <= 16 * 4 * 1024) DISTILL(0, 1024, 16);
    else DISTILL(0, 1024, 0);
  }
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
