// Generating tokens with a deployed subnet: the forward half of train.hip on rows that each continue a sequence, with attention over a
// paged cache of keys and values instead of over the batch.  Host orchestration, and the embedding of such rows.
#include <algorithm>
#include <cmath>

#include "nn.h"

namespace {

constexpr int kT = 256;

template <int BF> __device__ __forceinline__ float weight(const void *p, int64_t i) {
  return BF ? __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16) : static_cast<const float *>(p)[i];
}

// A wave per row: x = E[token] (+ P[position]), the position being the row's length less one; zeros for ids outside the vocabulary and for unused rows,
// which go on as rows of length 0 of sequence 0 (`used`, `of`): nothing is cached for them and they attend to nothing, but what they hold is a number
// all the same (a projection in fp32 forms tiles with results that are none in another way, rows of other sequences among them).  Bound by latency: one element a
// lane at a time, 13 us for one row of 2048, once a step.
template <int BF>
__global__ __launch_bounds__(kT) void decode_embed_kernel(const int32_t *tokens, const int32_t *seq, const int32_t *lens, int T, int n_seqs, int max_len, const void *E,
                                                          const void *P, float *x, int32_t *used, int32_t *of, int D, int vocab) {
  const int t = blockIdx.x * (kT / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= T) return;
  const int len = lens[t], s = seq ? seq[t] : t, tok = tokens[t];
  const bool on = len >= 1 && len <= max_len && (unsigned)s < (unsigned)n_seqs, known = on && (unsigned)tok < (unsigned)vocab;
  if (lane == 0) {
    used[t] = on ? len : 0;
    of[t] = on ? s : 0;
  }
  for (int c = lane; c < D; c += 64) {
    float v = known ? weight<BF>(E, (int64_t)tok * D + c) : 0.f;
    if (P && on) v += weight<BF>(P, (int64_t)(len - 1) * D + c);
    x[(int64_t)t * D + c] = v;
  }
}

// The pools of layer l lie one behind the other in the cache's storage, keys then values, the layers' behind each other: elements of a page, bytes of a pool
int64_t page_elems(const twist_ctx *ctx, const twist_subnet *sub, const twist_pages *pg, int l) {
  return (int64_t)sub->plan->layout.heads_sub[l] * pg->page_tokens * ctx->d.d_head;
}
size_t pool_bytes(const twist_ctx *ctx, const twist_subnet *sub, const twist_pages *pg, int l) {
  return align_up((size_t)pg->n_pages * page_elems(ctx, sub, pg, l) * ctx->esize(), 256);
}
size_t cache_size(const twist_ctx *ctx, const twist_subnet *sub, const twist_pages *pg) {
  size_t n = 0;
  for (int l = 0; l < ctx->d.n_layers; ++l) n += 2 * pool_bytes(ctx, sub, pg, l);
  return n;
}

struct Workspace {
  float *x[2], *stats, *scratch;
  int32_t *used, *of;
  void *h, *qkv, *q, *o, *gu, *a;
  size_t scratch_floats, bytes;
};

twist_status carve(twist_ctx *ctx, const twist_subnet *sub, const twist_pages *pg, int T, int max_len, char *base, Workspace &w) {
  const twist_model_desc &d = ctx->d;
  const SubLayout &L = sub->plan->layout;
  const size_t es = ctx->esize(), D = d.d_model;
  const int nf = d.act == TWIST_ACT_SWIGLU ? 2 : 1;
  size_t hd = 0, f = 0, off = 0;
  w.scratch_floats = 0;
  for (int l = 0; l < d.n_layers; ++l) {
    size_t n = 0;
    TW_TRY(twist_cache_attention_floats(ctx, pg, T, L.heads_sub[l], max_len, &n));
    w.scratch_floats = std::max(w.scratch_floats, n);
    hd = std::max(hd, (size_t)L.heads_sub[l] * d.d_head);
    f = std::max(f, (size_t)L.ffn_sub[l] * d.ffn_granule);
  }
  auto take = [&](size_t bytes) -> void * {
    char *p = base ? base + off : nullptr;
    off += align_up(bytes, 256);
    return p;
  };
  for (float *&x : w.x) x = static_cast<float *>(take(T * D * 4));
  w.stats = static_cast<float *>(take((size_t)T * 2 * 4));
  w.used = static_cast<int32_t *>(take((size_t)T * 4));
  w.of = static_cast<int32_t *>(take((size_t)T * 4));
  w.h = take(T * D * es);
  w.qkv = take(T * 3 * hd * es);
  w.q = d.use_rope ? take(T * hd * es) : nullptr;
  w.o = take(T * hd * es);
  w.gu = take(T * nf * f * es);
  w.a = take(T * f * es);
  w.scratch = static_cast<float *>(take(w.scratch_floats * 4));
  w.bytes = off;
  return TWIST_OK;
}

twist_status check_decode(twist_ctx *ctx, const char *who, const twist_subnet *sub, const twist_pages *pg, int T, int max_len) {
  const twist_model_desc &d = ctx->d;
  if (sub->ctx != ctx) TW_FAIL(ctx, TWIST_EINVAL, "%s: subnet belongs to another context", who);
  if (d.vocab < 1) TW_FAIL(ctx, TWIST_ESHAPE, "%s: needs a vocabulary", who);
  if (d.has_bias && d.act == TWIST_ACT_SWIGLU) TW_FAIL(ctx, TWIST_ESHAPE, "%s: gated FFN with biases is not supported", who);
  if (T < 1) TW_FAIL(ctx, TWIST_EINVAL, "%s: empty input", who);
  if (max_len < 1 || max_len > d.max_seq) TW_FAIL(ctx, TWIST_ESHAPE, "%s: max_len=%d is outside 1 .. max_seq=%d", who, max_len, d.max_seq);
  if ((int64_t)T * std::max(d.d_model, d.vocab) >= (1ll << 40)) TW_FAIL(ctx, TWIST_ESHAPE, "%s: batch too large", who);
  size_t n = 0;  // (checks the table, the widths and the head)
  for (int32_t heads : sub->plan->layout.heads_sub) TW_TRY(twist_cache_attention_floats(ctx, pg, T, heads, max_len, &n));
  return TWIST_OK;
}

}  // namespace

extern "C" twist_status twist_cache_bytes(twist_ctx *ctx, const twist_subnet *sub, const twist_pages *pages, size_t *bytes) {
  const char *who = "twist_cache_bytes";
  if (!ctx || !sub || !bytes) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  TW_TRY(check_decode(ctx, who, sub, pages, 1, 1));
  *bytes = cache_size(ctx, sub, pages);
  return TWIST_OK;
}

extern "C" twist_status twist_decode_workspace_bytes(twist_ctx *ctx, const twist_subnet *sub, const twist_pages *pages, int32_t T, int32_t max_len, size_t *bytes) {
  const char *who = "twist_decode_workspace_bytes";
  if (!ctx || !sub || !bytes) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  TW_TRY(check_decode(ctx, who, sub, pages, T, max_len));
  Workspace w;
  TW_TRY(carve(ctx, sub, pages, T, max_len, nullptr, w));
  *bytes = w.bytes;
  return TWIST_OK;
}

extern "C" twist_status twist_subnet_decode(twist_ctx *ctx, twist_subnet *sub, const int32_t *tokens, int32_t T, const int32_t *seq, const int32_t *lens,
                                            int32_t max_len, const twist_pages *pages, void *cache, size_t cache_bytes, void *workspace, size_t workspace_bytes,
                                            void *logits, int64_t ldl) {
  const char *who = "twist_subnet_decode";
  if (!ctx || !sub || !tokens || !lens || !cache || !workspace || !logits) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  TW_TRY(check_decode(ctx, who, sub, pages, T, max_len));
  const twist_model_desc &d = ctx->d;
  if (ldl < d.vocab) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of logits overlap", who);
  if (reinterpret_cast<uintptr_t>(cache) % 256 || reinterpret_cast<uintptr_t>(workspace) % 256) TW_FAIL(ctx, TWIST_ESHAPE, "%s: cache and workspace must be 256-byte aligned", who);
  const bool listed = seq || T > pages->n_seqs;  // (row t of sequence t needs no list)
  for (int32_t heads : sub->plan->layout.heads_sub) TW_TRY(twist_cache_attention_check(ctx, who, pages, T, heads, max_len, listed));  // (before anything is appended)
  const size_t need = cache_size(ctx, sub, pages);
  if (cache_bytes < need) TW_FAIL(ctx, TWIST_ESHAPE, "%s: cache of %zu bytes is smaller than the %zu needed", who, cache_bytes, need);
  Workspace w;
  TW_TRY(carve(ctx, sub, pages, T, max_len, static_cast<char *>(workspace), w));
  if (workspace_bytes < w.bytes) TW_FAIL(ctx, TWIST_ESHAPE, "%s: workspace of %zu bytes is smaller than the %zu needed", who, workspace_bytes, w.bytes);

  const SubLayout &L = sub->plan->layout;
  const int bf = d.dtype == TWIST_BF16, es = ctx->esize(), D = d.d_model, dh = d.d_head, rms = d.norm == TWIST_NORM_RMS;
  const int nf = d.act == TWIST_ACT_SWIGLU ? 2 : 1, scaled = sub->plan->scale_mode;
  const bool um = d.out_unit_major != 0;
  auto P = [&](const Slot &s) -> void * { return s.off < 0 ? nullptr : sub->params + s.off * es; };
  auto gemm = [&](GemmLayout lay, int N, int K, const void *A, const void *W, int64_t ldw, void *out, int64_t ldc, int out_f32, float alpha = 1.f,
                  const void *bias = nullptr, const float *residual = nullptr) {
    GemmEpilogue e;
    e.alpha = alpha; e.bias = bias; e.residual = residual; e.out = out; e.out_f32 = out_f32;
    return twist_gemm(ctx, bf, lay, T, N, K, A, K, W, ldw, ldc, e);
  };
  const dim3 grid((T + kT / 64 - 1) / (kT / 64));
  if (bf) hipLaunchKernelGGL((decode_embed_kernel<1>), grid, dim3(kT), 0, ctx->stream, tokens, seq, lens, T, pages->n_seqs, max_len, P(L.global[TWIST_TOK_EMBED]),
                             P(L.global[TWIST_POS_EMBED]), w.x[0], w.used, w.of, D, d.vocab);
  else hipLaunchKernelGGL((decode_embed_kernel<0>), grid, dim3(kT), 0, ctx->stream, tokens, seq, lens, T, pages->n_seqs, max_len, P(L.global[TWIST_TOK_EMBED]),
                          P(L.global[TWIST_POS_EMBED]), w.x[0], w.used, w.of, D, d.vocab);
  TW_HIP(ctx, hipGetLastError());
  const int32_t *of = listed ? w.of : nullptr;
  char *k = static_cast<char *>(cache), *v;
  for (int l = 0; l < d.n_layers; ++l, k = v + pool_bytes(ctx, sub, pages, l - 1)) {
    const int Hs = L.heads_sub[l], HD = Hs * dh, F = L.ffn_sub[l] * d.ffn_granule;
    const float c_a = scaled ? sqrtf((float)d.n_heads / (float)Hs) : 1.f, c_f = scaled ? sqrtf((float)ctx->n_ffn_units() / (float)L.ffn_sub[l]) : 1.f;
    const int64_t page = page_elems(ctx, sub, pages, l);
    v = k + pool_bytes(ctx, sub, pages, l);
    TW_TRY(twist_norm_fwd(ctx, bf, rms, w.x[0], P(L.at(l, TWIST_NORM1_W)), P(L.at(l, TWIST_NORM1_B)), w.h, w.stats, T, D, d.norm_eps));
    TW_TRY(gemm(GEMM_NT, 3 * HD, D, w.h, P(L.at(l, TWIST_WQ)), D, w.qkv, 3 * HD, 0, 1.f, P(L.at(l, TWIST_BQ))));
    TW_TRY(twist_cache_append_raw(ctx, pages, k, v, page, w.qkv, 3 * HD, T, Hs, of, w.used, w.q, HD));
    TW_TRY(twist_cache_attention_raw(ctx, pages, k, v, page, w.q ? w.q : w.qkv, w.q ? HD : 3 * HD, T, Hs, of, w.used, max_len, w.o, HD, nullptr, w.scratch,
                                     w.scratch_floats));
    TW_TRY(gemm(um ? GEMM_NN : GEMM_NT, D, HD, w.o, P(L.at(l, TWIST_WO)), um ? D : HD, w.x[1], D, 1, c_a, P(L.at(l, TWIST_BO)), w.x[0]));
    TW_TRY(twist_norm_fwd(ctx, bf, rms, w.x[1], P(L.at(l, TWIST_NORM2_W)), P(L.at(l, TWIST_NORM2_B)), w.h, w.stats, T, D, d.norm_eps));
    if (nf == 1) {
      GemmEpilogue e;
      e.bias = P(L.at(l, TWIST_B_UP)); e.out = w.gu; e.act_out = w.a; e.act = d.act; e.act_only = true;
      TW_TRY(twist_gemm(ctx, bf, GEMM_NT, T, F, D, w.h, D, P(L.at(l, TWIST_W_UP)), D, F, e));
    } else {
      TW_TRY(gemm(GEMM_NT, 2 * F, D, w.h, P(L.at(l, TWIST_W_GATE)), D, w.gu, 2 * F, 0));
      TW_TRY(twist_act_fwd(ctx, bf, d.act, w.gu, w.a, T, F));
    }
    TW_TRY(gemm(um ? GEMM_NN : GEMM_NT, D, F, w.a, P(L.at(l, TWIST_W_DOWN)), um ? D : F, w.x[0], D, 1, c_f, P(L.at(l, TWIST_B_DOWN)), w.x[1]));
  }
  TW_TRY(twist_norm_fwd(ctx, bf, rms, w.x[0], P(L.global[TWIST_FINAL_NORM_W]), P(L.global[TWIST_FINAL_NORM_B]), w.h, w.stats, T, D, d.norm_eps));
  return gemm(GEMM_NT, d.vocab, D, w.h, P(d.tied_head ? L.global[TWIST_TOK_EMBED] : L.global[TWIST_LM_HEAD]), D, logits, ldl, 0);
}
