// The paged cache of keys and values behind twist_subnet_decode: appending to it, with the rotary embedding on the way, and attention of
// new tokens over it.
#include "nn.h"

namespace {

constexpr int kT = 256;

template <int BF> struct El;
template <> struct El<0> {
  static __device__ __forceinline__ float ld(const void *p, int64_t i) { return static_cast<const float *>(p)[i]; }
  static __device__ __forceinline__ void st(void *p, int64_t i, float v) { static_cast<float *>(p)[i] = v; }
};
template <> struct El<1> {
  static __device__ __forceinline__ float ld(const void *p, int64_t i) {
    return __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
  }
  static __device__ __forceinline__ void st(void *p, int64_t i, float v) {
    uint32_t u = __float_as_uint(v);
    if ((u & 0x7fffffffu) > 0x7f800000u) u = (u >> 16) | 0x40u;
    else { u += 0x7fffu + ((u >> 16) & 1u); u >>= 16; }
    static_cast<uint16_t *>(p)[i] = (uint16_t)u;
  }
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// the page table as the kernels use it
struct Pages {
  const int32_t *table;
  int64_t ld;
  int32_t n_seqs, max_pages, n_pages, shift;  // page_tokens = 1 << shift
};

// element offset of head h of token p of sequence s, in pools of Hs heads of dh; -1: the sequence has no such page
__device__ __forceinline__ int64_t place(const Pages &pg, int64_t page_stride, int s, int p, int h, int dh) {
  const int i = p >> pg.shift;
  if (i >= pg.max_pages) return -1;
  const int page = pg.table[s * pg.ld + i];
  if ((unsigned)page >= (unsigned)pg.n_pages) return -1;
  return page * page_stride + (((int64_t)h << pg.shift) + (p & ((1 << pg.shift) - 1))) * dh;
}

// ------------------------------------------------------------------------------------------- append
// cos and sin of the rotary embedding's angle of pair i at position p, p theta^(-2i/dh): `turns` = theta^(-2i/dh) / 2 pi, so that the whole
// turns come off exactly in fp64 and what is left, at most half a turn, keeps an fp32's precision at any position.
__device__ __forceinline__ void rotation(int p, double turns, float &c, float &s) {
  const double t = (double)p * turns;
  sincospif(2.f * (float)(t - rint(t)), &s, &c);
}

struct Turns { double f[128]; };  // theta^(-2i/dh) / 2 pi

// A thread per (row, head, pair (i, i + dh/2)) with rotation, per (row, head, element) without.
template <int BF, bool ROPE>
__global__ __launch_bounds__(kT) void append_plain_kernel(Pages pg, void *k, void *v, int64_t page_stride, const void *qkv, int64_t ld, int Hs, int dh,
                                                          const int32_t *seq, const int32_t *lens, void *q_out, int64_t ldq, Turns turns, int64_t total) {
  const int64_t i = (int64_t)blockIdx.x * kT + threadIdx.x;
  if (i >= total) return;
  const int n = ROPE ? dh / 2 : dh;
  const int f = (int)(i % n);
  const int64_t r = i / n;
  const int h = (int)(r % Hs);
  const int t = (int)(r / Hs), p = lens[t] - 1, s = seq ? seq[t] : t;
  if (p < 0 || (unsigned)s >= (unsigned)pg.n_seqs) return;
  const int64_t HD = (int64_t)Hs * dh, in = t * ld + (int64_t)h * dh + f, out = t * ldq + (int64_t)h * dh + f, at = place(pg, page_stride, s, p, h, dh);
  if (!ROPE) {
    if (q_out) El<BF>::st(q_out, out, El<BF>::ld(qkv, in));
    if (at < 0) return;
    El<BF>::st(k, at + f, El<BF>::ld(qkv, in + HD));
    El<BF>::st(v, at + f, El<BF>::ld(qkv, in + 2 * HD));
    return;
  }
  float c, sn;
  rotation(p, turns.f[f], c, sn);
  if (q_out) {
    const float a = El<BF>::ld(qkv, in), b = El<BF>::ld(qkv, in + n);
    El<BF>::st(q_out, out, a * c - b * sn);
    El<BF>::st(q_out, out + n, b * c + a * sn);
  }
  if (at < 0) return;
  const float a = El<BF>::ld(qkv, in + HD), b = El<BF>::ld(qkv, in + HD + n);
  El<BF>::st(k, at + f, a * c - b * sn);
  El<BF>::st(k, at + f + n, b * c + a * sn);
  El<BF>::st(v, at + f, El<BF>::ld(qkv, in + 2 * HD));
  El<BF>::st(v, at + f + n, El<BF>::ld(qkv, in + 2 * HD + n));
}

// ------------------------------------------------------------------------------------------- attention
constexpr int kE = 4;  // d_head <= 64 * kE

// A wave per (row, head), one key at a time, running maximum and sum of the softmax.
template <int BF>
__global__ __launch_bounds__(kT) void cache_attention_plain_kernel(Pages pg, const void *k, const void *v, int64_t page_stride, const void *q, int64_t ldq, int T,
                                                                   int Hs, int dh, const int32_t *seq, const int32_t *lens, int max_len, void *o, int64_t ldo,
                                                                   float *lse, float scale) {
  const int64_t w = (int64_t)blockIdx.x * (kT / 64) + (threadIdx.x >> 6);
  if (w >= (int64_t)T * Hs) return;
  const int h = (int)(w % Hs), t = (int)(w / Hs), lane = threadIdx.x & 63, s = seq ? seq[t] : t, len = min(lens[t], max_len);
  if (lens[t] < 0 || (unsigned)s >= (unsigned)pg.n_seqs) return;
  float x[kE], acc[kE];
#pragma unroll
  for (int j = 0; j < kE; ++j) { const int e = lane + 64 * j; x[j] = e < dh ? El<BF>::ld(q, t * ldq + (int64_t)h * dh + e) : 0.f; acc[j] = 0.f; }
  float m = -INFINITY, l = 0.f;
  bool any = false;
  for (int p = 0; p < len; ++p) {
    const int64_t at = place(pg, page_stride, s, p, h, dh);
    if (at < 0) continue;
    any = true;
    float d = 0.f;
#pragma unroll
    for (int j = 0; j < kE; ++j) { const int e = lane + 64 * j; if (e < dh) d += x[j] * El<BF>::ld(k, at + e); }
    d = wave_sum(d) * scale;
    const float mn = fmaxf(m, d), ref = mn == -INFINITY ? 0.f : mn;  // scores of -infinity have no weight beside others
    const float c = expf(m - ref), e1 = expf(d - ref);
    l = l * c + e1;
#pragma unroll
    for (int j = 0; j < kE; ++j) { const int e = lane + 64 * j; if (e < dh) acc[j] = acc[j] * c + e1 * El<BF>::ld(v, at + e); }
    m = mn;
  }
#pragma unroll
  for (int j = 0; j < kE; ++j) { const int e = lane + 64 * j; if (e < dh) El<BF>::st(o, t * ldo + (int64_t)h * dh + e, any ? acc[j] / l : 0.f); }
  if (lse && lane == 0) lse[(int64_t)t * Hs + h] = m + logf(l);
}

twist_status check_pages(twist_ctx *ctx, const char *who, const twist_pages *p) {
  if (!p || !p->table) TW_FAIL(ctx, TWIST_EINVAL, "%s: null page table", who);
  if (p->n_seqs < 1 || p->max_pages < 1 || p->n_pages < 1) TW_FAIL(ctx, TWIST_EINVAL, "%s: a cache has at least one sequence and one page", who);
  if (p->ld_table < p->max_pages) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of the page table overlap", who);
  if (p->page_tokens < 1 || p->page_tokens > 4096 || (p->page_tokens & (p->page_tokens - 1)))
    TW_FAIL(ctx, TWIST_ESHAPE, "%s: page_tokens=%d is not a power of two up to 4096", who, p->page_tokens);
  if ((int64_t)p->max_pages * p->page_tokens > INT32_MAX) TW_FAIL(ctx, TWIST_ESHAPE, "%s: positions beyond 2^31", who);
  return TWIST_OK;
}

// the arguments that both calls have
twist_status check_cache(twist_ctx *ctx, const char *who, const twist_pages *p, int64_t page_stride, int T, int Hs) {
  TW_TRY(check_pages(ctx, who, p));
  const int64_t dh = ctx->d.d_head;
  if (T < 1 || Hs < 1) TW_FAIL(ctx, TWIST_EINVAL, "%s: empty input", who);
  if (dh > 64 * kE) TW_FAIL(ctx, TWIST_ESHAPE, "%s: d_head=%lld above %d is not supported", who, (long long)dh, 64 * kE);
  if ((int64_t)T * Hs > (int64_t)1 << 24 || Hs > 65535) TW_FAIL(ctx, TWIST_ESHAPE, "%s: %d rows of %d heads are too many for one call", who, T, Hs);
  if (page_stride < Hs * dh * p->page_tokens) TW_FAIL(ctx, TWIST_ESHAPE, "%s: page_stride=%lld is less than a page", who, (long long)page_stride);
  return TWIST_OK;
}

Pages device_pages(const twist_pages *p) {
  return {p->table, p->ld_table, p->n_seqs, p->max_pages, p->n_pages, __builtin_ctz((unsigned)p->page_tokens)};
}

}  // namespace

extern "C" twist_status twist_cache_append_raw(twist_ctx *ctx, const twist_pages *pages, void *k, void *v, int64_t page_stride, const void *qkv, int64_t ld,
                                               int32_t T, int32_t Hs, const int32_t *seq, const int32_t *lens, void *q_out, int64_t ldq) {
  const char *who = "twist_cache_append_raw";
  if (!ctx || !k || !v || !qkv || !lens) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  TW_TRY(check_cache(ctx, who, pages, page_stride, T, Hs));
  const int dh = ctx->d.d_head;
  const int64_t HD = (int64_t)Hs * dh;
  if (ld < 3 * HD || (q_out && ldq < HD)) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows overlap", who);
  const Pages pg = device_pages(pages);
  Turns turns;
  for (int i = 0; i < 128; ++i) turns.f[i] = ctx->rope_turns[i];
  const int rope = ctx->d.use_rope;
  const int64_t total = (int64_t)T * Hs * (rope ? dh / 2 : dh);
  const dim3 grid((unsigned)((total + kT - 1) / kT));
#define APPEND(BF, R) hipLaunchKernelGGL((append_plain_kernel<BF, R>), grid, dim3(kT), 0, ctx->stream, pg, k, v, page_stride, qkv, ld, Hs, dh, seq, lens, q_out, ldq, turns, total)
  if (ctx->d.dtype == TWIST_BF16) { if (rope) APPEND(1, true); else APPEND(1, false); }
  else { if (rope) APPEND(0, true); else APPEND(0, false); }
#undef APPEND
  TW_HIP(ctx, hipGetLastError());
  return TWIST_OK;
}

extern "C" twist_status twist_cache_attention_floats(twist_ctx *ctx, const twist_pages *pages, int32_t T, int32_t Hs, int32_t max_len, size_t *floats) {
  const char *who = "twist_cache_attention_floats";
  if (!ctx || !floats) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  TW_TRY(check_cache(ctx, who, pages, INT64_MAX, T, Hs));
  if (max_len < 1) TW_FAIL(ctx, TWIST_EINVAL, "%s: max_len=%d", who, max_len);
  *floats = 0;
  return TWIST_OK;
}

extern "C" twist_status twist_cache_attention_raw(twist_ctx *ctx, const twist_pages *pages, const void *k, const void *v, int64_t page_stride, const void *q,
                                                  int64_t ldq, int32_t T, int32_t Hs, const int32_t *seq, const int32_t *lens, int32_t max_len, void *o,
                                                  int64_t ldo, float *lse, float *scratch, size_t scratch_floats) {
  const char *who = "twist_cache_attention_raw";
  if (!ctx || !k || !v || !q || !lens || !o) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  TW_TRY(check_cache(ctx, who, pages, page_stride, T, Hs));
  size_t need = 0;
  TW_TRY(twist_cache_attention_floats(ctx, pages, T, Hs, max_len, &need));
  if (need && !scratch) TW_FAIL(ctx, TWIST_EINVAL, "%s: null scratch", who);
  if (scratch_floats < need) TW_FAIL(ctx, TWIST_ESHAPE, "%s: scratch of %zu floats is smaller than the %zu needed", who, scratch_floats, need);
  const int dh = ctx->d.d_head;
  const int64_t HD = (int64_t)Hs * dh;
  if (ldq < HD || ldo < HD) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows overlap", who);
  const Pages pg = device_pages(pages);
  const int64_t cap = (int64_t)pages->max_pages * pages->page_tokens;
  if (max_len > cap) max_len = (int32_t)cap;
  const dim3 grid((unsigned)(((int64_t)T * Hs + 3) / 4));
  const float scale = 1.f / sqrtf((float)dh);
  if (ctx->d.dtype == TWIST_BF16)
    hipLaunchKernelGGL((cache_attention_plain_kernel<1>), grid, dim3(kT), 0, ctx->stream, pg, k, v, page_stride, q, ldq, T, Hs, dh, seq, lens, max_len, o, ldo, lse, scale);
  else
    hipLaunchKernelGGL((cache_attention_plain_kernel<0>), grid, dim3(kT), 0, ctx->stream, pg, k, v, page_stride, q, ldq, T, Hs, dh, seq, lens, max_len, o, ldo, lse, scale);
  TW_HIP(ctx, hipGetLastError());
  return TWIST_OK;
}
