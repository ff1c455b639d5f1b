// The loss of a student's logits against a teacher's top logits and the targets, with its gradient.
#include <cfloat>
#include <type_traits>

#include "nn.h"
#include "row.h"

namespace {

constexpr int kTop = 1024;  // the longest list
constexpr float kLog2e = 1.44269504f;

template <int BF> __device__ __forceinline__ void store_piece(char *p, const float *g) {
  u32x4v u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    if (BF) u[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{g[2 * i % Piece<BF>::N], g[(2 * i + 1) % Piece<BF>::N]}), b2));
    else u[i] = __float_as_uint(g[i]);
  }
  __builtin_memcpy(p, &u, 16);
}

// exp(x) in 32 bits: the exponent's rounding, which a large one would multiply, taken care of
__device__ __forceinline__ float exp_f32(double x) {
  const double y = x * 1.4426950408889634;
  if (y <= -200.0) return 0.f;
  const float h = (float)y;
  return __builtin_amdgcn_exp2f(h) * fmaf((float)(y - h), 0.69314718f, 1.f);
}

// A row a workgroup.  The row's tokens are the teacher's (the set) and the others, whose share of the distribution is formed from themselves and not as what the set leaves: it
// may be next to nothing, or all but everything.  With tau the temperature, p and q over the set and over the others together (P, Q of them), the gradient of KL(q || p) is
// (p_i - q_i) / tau in the set and p_i (P - Q) / P / tau outside it.
// Bound by memory: the row is read once and its gradient written once (64 entries, 8192 x 50257 bf16: 342 us, 4.8 TB/s, the rate of a copy; 1024 x 50257 fp32, one row a CU at a
// time: 112 us, 3.7).  It stays in registers as it came (NV pieces of 16 bytes a thread; bf16 with 16 of them spills one register), the set's columns as -infinity, so that they
// weigh nothing in the others' sums; their own gradients, a thread each and in 64 bits where they meet a logarithm, are stored over the others' behind a barrier.  Rows that NT
// threads cannot hold, NV = 0, are read three times (1024 x 131072: bf16 212 us, 2.5 TB/s of what one pass would move, fp32 357, 3.0).
// Pieces begin where the gradient's row is aligned, which is where the logits' is as a rule (rows of an odd vocabulary start anywhere; 8192 x 50257 bf16 from any element on
// 554 us, all rows aligned 440); the columns before and behind them are a thread's each.
template <int BF, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void distill_kernel(const char *logits, int64_t ld, const int32_t *targets, int V, twist_teacher te, char *grads, int64_t ldg, int64_t pad, float inv_T,
                                                        float *rowloss) {
  using P16 = Piece<BF>;
  constexpr int N = P16::N, ES = P16::ES, NW = NT / 64, WORDS = NV ? NV * NT * N / 32 + 1 : (1 << 15) + 1;
  __shared__ uint32_t in_set[WORDS];  // a bit a column, the first of a piece on a byte (fp32: half a byte)
  __shared__ int32_t id[kTop];
  __shared__ float logit[kTop];
  __shared__ double weight[kTop], part[kTop];  // the teacher's weights against its largest, and their exponents
  __shared__ float most[3][NW], sums[2][NW];
  __shared__ double set_sums[4][NW];
  __shared__ int twice;
  const int t = blockIdx.x, tid = threadIdx.x, k = te.k, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const device_bytes row = (device_bytes)(logits + (int64_t)t * ld * ES);
  char *out = grads + (int64_t)t * ldg * ES;
  const int head = min(V, (int)(-(reinterpret_cast<uintptr_t>(out) / ES) & (N - 1)));
  const int pieces = (V - head) / N, mine = pieces - 64 * wave;  // u NT >= mine: the wave's piece u lies beyond the row
  const int ends = V - pieces * N, end = tid < head ? tid : pieces * N + tid;  // columns that are in no piece, and the thread's
  const device_bytes first = row + head * ES;
  char *first_out = out + head * ES;
  // what the first of the list need, and the row
  const int64_t list = t * te.ld;
  const int id0 = tid < k ? te.ids[list + tid] : -1;
  const float value0 = tid < k ? te.values[list + tid] : 0.f;
  const int tgt = te.weight < 1.f ? targets[t] : -1;
  const bool aimed = (unsigned)tgt < (unsigned)V;
  const float rest = te.rest ? te.rest[t] : -INFINITY;
  P16 x[NV ? NV : 1];  // (as a Row's, but that the list's columns are taken out of it, also of pieces that are read again)
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    x[u].u = P16::none();
    if (u * NT + tid < pieces) x[u].load(first + (int64_t)(u * NT + tid) * 16);
  }
  float xl = tid < ends ? load1<BF>(row, end) : -INFINITY;
  const float aim = aimed ? load1<BF>(row, tgt) : 0.f;
  const double tau = te.temperature, inv_tau = 1.0 / tau;
  for (int i = tid; i < (V + N + 31) / 32; i += NT) in_set[i] = 0;
  if (tid == 0) twice = 0;
  auto bit = [&](int c) { return c - head + N; };  // of a column, in the table
  __syncthreads();
  float top_value = -INFINITY, top_set = -INFINITY;  // largest of the teacher's values, and of the student's in the set
  for (int j = tid; j < k; j += NT) {
    const int c = j == tid ? id0 : te.ids[list + j];
    const bool on = (unsigned)c < (unsigned)V;
    id[j] = on ? c : -1;
    if (!on) continue;
    const float s = load1<BF>(row, c);
    if (atomicOr(&in_set[bit(c) / 32], 1u << (bit(c) & 31)) >> (bit(c) & 31) & 1) twice = 1;
    logit[j] = s;
    top_set = fmaxf(top_set, s);
    const float value = j == tid ? value0 : te.values[list + j];
    part[j] = value * inv_tau;
    top_value = fmaxf(top_value, value);
  }
  if (64 * wave < k) {
    top_value = wave_max(top_value);
    top_set = wave_max(top_set);
  }
  if (lane == 0) { most[0][wave] = top_value; most[1][wave] = top_set; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) { top_value = fmaxf(top_value, most[0][w]); top_set = fmaxf(top_set, most[1][w]); }
  const double top_t = fmax(top_value * inv_tau, (double)rest);  // (a finite value over the temperature may be beyond fp32)
  const bool taught = te.weight > 0.f && top_t > -INFINITY;
  if (!taught && !aimed) {
    const float zeros[N] = {};
    for (int v = tid; v < pieces; v += NT) store_piece<BF>(first_out + (int64_t)v * 16, zeros);
    if (tid < ends) store1<BF>(out, end, 0.f);
    for (int64_t c = V + tid; c < pad; c += NT) store1<BF>(out, c, 0.f);
    if (tid == 0) rowloss[t] = 0.f;
    return;
  }
  auto bits_of = [&](int v) {  // of a piece's columns in the set
    const uint32_t b = reinterpret_cast<const uint8_t *>(in_set)[N == 8 ? v + 1 : (v + 1) / 2];
    return N == 8 ? b : b >> ((v + 1) % 2 * 4) & 15u;
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
        y.load(first + (int64_t)v * 16);
        y.clear(bits_of(v));
        f(y, v);
      }
    }
  };
#pragma unroll
  for (int u = 0; u < NV; ++u)
    if (u * NT + tid < pieces) {
      const uint32_t b = bits_of(u * NT + tid);
      if (b) x[u].clear(b);
    }
  if (tid < ends && in_set[bit(end) / 32] >> (bit(end) & 31) & 1) xl = -INFINITY;
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
      part[j] -= top_t;
      weight[j] = taught ? exp(part[j]) : 0.0;
    }
  const double rest_weight = taught && rest > -INFINITY ? exp((double)rest - top_t) : 0.0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) other = fmaxf(other, most[2][w]);
  if (twice) {  // (every entry is compared with every other: 2048 x 32000 bf16, 64 entries 63 -> 73 us, 256 70 -> 99, 1024 106 -> 547)
    constexpr int M = (kTop + NT - 1) / NT;
    double sum[M];
    bool first_of[M];
#pragma unroll
    for (int u = 0; u < M; ++u) {
      const int j = u * NT + tid;
      sum[u] = 0.0;
      first_of[u] = j < k && id[j] >= 0;
      if (first_of[u])
        for (int i = 0; i < k; ++i)
          if (id[i] == id[j]) {
            sum[u] += weight[i];
            first_of[u] = first_of[u] && i >= j;
          }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < M; ++u) {
      const int j = u * NT + tid;
      if (j < k && !first_of[u]) id[j] = -1;
      else if (j < k && sum[u] != weight[j]) {
        weight[j] = sum[u];
        part[j] = log(sum[u]);
      }
    }
  }
  const float ref = other > -INFINITY ? other : 0.f, m = fmaxf(top_set, other);
  // Sums over the others against their largest, and over the set against the row's.  Exponentials of (v - ref) / tau, and of v - ref: the same or only one of them asked for
  // (mode 0), squares (temperature 2: 1; 4: 2), or an exponential each (3).  8192 x 50257 bf16, both asked for: at temperature 2 341 us, at 1.5 or 3 383 (with the choice made
  // for every element 487); the teacher's alone, at 1.5, 318
  const float c1 = kLog2e, ct = fminf((float)(kLog2e * inv_tau), FLT_MAX), c = taught ? ct : c1;
  const int mode = !(taught && aimed) || te.temperature == 1.f ? 0 : te.temperature == 2.f ? 1 : te.temperature == 4.f ? 2 : 3;
  auto exps = [&](auto how, float v, auto f) {  // f(first, second)
    const float d = v - ref, a = __builtin_amdgcn_exp2f(d * c);
    if (how == 0) f(a, a);
    else if (how == 1) f(a, a * a);
    else if (how == 2) f(a, (a * a) * (a * a));
    else f(a, __builtin_amdgcn_exp2f(d * c1));
  };
  auto in_mode = [&](auto f) {
    if (mode == 0) f(std::integral_constant<int, 0>{});
    else if (mode == 1) f(std::integral_constant<int, 1>{});
    else if (mode == 2) f(std::integral_constant<int, 2>{});
    else f(std::integral_constant<int, 3>{});
  };
  const double down = other > -INFINITY ? (double)other - m : 0.0;
  const float w1 = (1.f - te.weight) * inv_T, wt = te.weight * te.temperature * inv_T;
  double others1 = 0.0, others = 0.0, set1 = 0.0, set = 0.0, qs = 0.0, kl = 0.0;
  float iz1, iz, izq, a1, as;
  auto slope = [&](auto how, float a, float b) { return how ? fmaf(b, a1, a * as) : a * as; };
  in_mode([&](auto how) {
    float s1 = 0.f, st = 0.f;
    auto add = [&](float a, float b) {
      st += a;
      if (how) s1 += b;
    };
    exps(how, xl, add);
    each([&](const P16 &y, int) {
#pragma unroll
      for (int e = 0; e < N; ++e) exps(how, y[e], add);
    });
    for (int j = tid; j < k; j += NT)
      if (id[j] >= 0) {
        const double d = (double)logit[j] - m;
        if (aimed) set1 += exp_f32(d);
        if (taught) set += exp(d * inv_tau);
        qs += weight[j];
        if (weight[j] != 0.0) kl += weight[j] * (part[j] - d * inv_tau);
      }
    st = wave_add(st);
    s1 = how ? wave_add(s1) : st;
    if (64 * wave < k) { set1 = wave_add(set1); set = wave_add(set); qs = wave_add(qs); kl = wave_add(kl); }
    if (lane == 0) {
      sums[0][wave] = s1; sums[1][wave] = st;
      set_sums[0][wave] = set1; set_sums[1][wave] = set; set_sums[2][wave] = qs; set_sums[3][wave] = kl;
    }
    __syncthreads();
    set1 = set = qs = kl = 0.0;
#pragma unroll 1
    for (int w = 0; w < NW; ++w) {
      others1 += sums[0][w]; others += sums[1][w];
      if (64 * w < k) { set1 += set_sums[0][w]; set += set_sums[1][w]; qs += set_sums[2][w]; kl += set_sums[3][w]; }
    }
    const float down1 = __expf((float)down), others_m = (float)others * __builtin_amdgcn_exp2f((float)down * ct);
    iz1 = 1.f / fmaf((float)others1, down1, (float)set1);
    iz = 1.f / (others_m + (float)set);
    izq = 1.f / (float)(qs + rest_weight);
    const float Q = taught ? (float)rest_weight * izq : 0.f, P = others_m * iz;
    // the others' gradient is their share of each other times P - Q, which is what the set's probabilities differ by
    const float more = Q < 0.5f ? P - Q : (float)qs * izq - (float)set * iz, at = taught && others > 0.0 ? wt * more / (float)others : 0.f;
    a1 = aimed ? w1 * down1 * iz1 : 0.f;
    as = how ? at : a1 + at;
    each([&](const P16 &y, int v) {
      float g[N];
#pragma unroll
      for (int e = 0; e < N; ++e) exps(how, y[e], [&](float a, float b) { g[e] = slope(how, a, b); });
      if (v < pieces) store_piece<BF>(first_out + (int64_t)v * 16, g);
    });
    if (tid < ends) exps(how, xl, [&](float a, float b) { store1<BF>(out, end, slope(how, a, b)); });
  });
  for (int64_t c = V + tid; c < pad; c += NT) store1<BF>(out, c, 0.f);
  if (wave == NW - 1) {
    // the row's loss, in 64 bits: the share of one of two amounts is formed from their quotient, so that it is as exact near 1 as far from it.  A lane each for what would be one
    // call behind the other.
    auto of = [](double v, int from) { return __shfl(v, from, 64); };
    const double e = exp(lane == 0 ? down * inv_tau : down), rm = others * of(e, 0), r1 = others1 * of(e, 1) + set1, whole = rm + set, qall = qs + rest_weight;
    const double a = lane == 0 ? rm : rest_weight, b = lane == 0 ? set : qs, ratio = b < a ? b / a : a / b;  // (lanes 0 and 1)
    const double l = log(lane == 0 ? whole : lane == 1 ? qall : lane == 2 ? r1 : lane == 3 ? others : lane == 4 ? rm / set : rest_weight / qs), l1 = log1p(ratio);
    const double share = rm > 0.0 ? -of(l1, 0) + (set < rm ? 0.0 : of(l, 4)) : down * inv_tau + (others > 0.0 ? of(l, 3) : -INFINITY) - of(l, 0);
    const double theirs = -of(l1, 1) + (qs < rest_weight ? 0.0 : of(l, 5));
    double loss = aimed ? (1.0 - (double)te.weight) * (of(l, 2) - ((double)aim - m)) : 0.0;
    if (taught) {
      kl += qs != 0.0 ? qs * (of(l, 0) - of(l, 1)) : 0.0;
      if (rest_weight != 0.0) kl += rest_weight * (theirs - share);
      loss += (double)te.weight * tau * tau * (kl / qall);
    }
    if (lane == 0) rowloss[t] = (float)loss;
  }
  __syncthreads();  // (the set's gradients take the places of what was written above, and so does the target's)
  for (int j = tid; j < k; j += NT)
    if (id[j] >= 0) {
      const double d = (double)logit[j] - m;
      float g = taught ? wt * (exp_f32(d * inv_tau) * iz - (float)weight[j] * izq) : 0.f;
      if (aimed) g += w1 * (exp_f32(d) * iz1 - (id[j] == tgt ? 1.f : 0.f));
      store1<BF>(out, id[j], g);
    }
  if (tid == NT - 1 && aimed && !(in_set[bit(tgt) / 32] >> (bit(tgt) & 31) & 1))
    in_mode([&](auto how) { exps(how, aim, [&](float a, float b) { store1<BF>(out, tgt, slope(how, a, b) - w1); }); });
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
  // The fewest threads whose registers hold a row, so that a CU has several rows (64 entries, bf16: 256 x 32000 19.8 us with 256 threads and 18.3 with 1024, but 1024 x 32000 39
  // and 57, 4096 x 32000 121 and 212; 4096 x 50257 192 with 512, 290 with 1024; fp32 4096 x 16384 122 with 256, 177 with 1024, 4096 x 32000 207 with 512, 277 with 1024)
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
