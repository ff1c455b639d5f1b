// The paged cache of keys and values behind twist_subnet_decode: appending to it, with the rotary embedding on the way, and attention of
// new tokens over it.
#include <algorithm>

#include "nn.h"

namespace {

constexpr int kT = 256;

template <int BF> __device__ __forceinline__ void store1(void *p, int64_t i, float v) {
  if (BF) static_cast<__bf16 *>(p)[i] = (__bf16)v;
  else static_cast<float *>(p)[i] = v;
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

// theta^(-2i/dh) / 2 pi for pair i < 128, as a product (whose rounding, 2^-53, is nothing at any position).  All 128 as kernel arguments took the host 0.8 us more.
struct Turns {
  double coarse[8], fine[16];
  __device__ __forceinline__ double of(int i) const { return coarse[i >> 4] * fine[i & 15]; }
};

// BYTES (16 to an element's) of consecutive elements in registers
template <int BYTES> struct Vec;
template <> struct Vec<16> { typedef uint32_t T __attribute__((ext_vector_type(4))); };
template <> struct Vec<8> { typedef uint32_t T __attribute__((ext_vector_type(2))); };
template <> struct Vec<4> { typedef uint32_t T; };
template <> struct Vec<2> { typedef uint16_t T; };
template <int BF, int BYTES> struct Elems {
  static constexpr int N = BYTES / (BF ? 2 : 4);
  typename Vec<BYTES>::T raw;
  __device__ __forceinline__ void load(const void *p, int64_t i) { raw = *reinterpret_cast<const typename Vec<BYTES>::T *>(static_cast<const char *>(p) + i * (BF ? 2 : 4)); }
  __device__ __forceinline__ void store(void *p, int64_t i) const { *reinterpret_cast<typename Vec<BYTES>::T *>(static_cast<char *>(p) + i * (BF ? 2 : 4)) = raw; }
  __device__ __forceinline__ float get(int j) const {
    float v;
    if (BF) v = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(&raw)[j] << 16);
    else v = reinterpret_cast<const float *>(&raw)[j];
    return v;
  }
  __device__ __forceinline__ void set(const float *v) {  // (two bf16 to an instruction)
    if constexpr (BF) {
      typedef __bf16 To __attribute__((ext_vector_type(N)));
      typedef float From __attribute__((ext_vector_type(N)));
      From x;
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = v[j];
      raw = __builtin_bit_cast(typename Vec<BYTES>::T, __builtin_convertvector(x, To));
    } else {
      __builtin_memcpy(&raw, v, BYTES);
    }
  }
};

constexpr int kAngles = 1024;  // (row, pair) angles of a workgroup
constexpr int kAppendRows = 16;

// Bound by copying (every value read and written once), by a launch's latency for few rows.  A workgroup takes `rows` rows; the angles, the same for all heads,
// are formed once in LDS (left to every thread they took 1.5 times as long as the copying) while the first values are on their way; a
// thread then turns BYTES of the first half of a head against the same of the second, for q and k, and copies v.  us in a graph, heads of 128 in bf16: 1 row of 16
// 2.5 (an empty kernel 1.7), 72 rows of 16 2.8, 512 of 16 4.0, 8192 of 32 77 (5.2 TB/s).
template <int BF, int BYTES, bool ROPE>
__global__ __launch_bounds__(kT) void append_kernel(Pages pg, void *k, void *v, int64_t page_stride, const void *qkv, int64_t ld, int T, int Hs, int dh,
                                                    const int32_t *seq, const int32_t *lens, void *q_out, int64_t ldq, Turns turns, int rows) {
  using E = Elems<BF, BYTES>;
  constexpr int N = E::N, HALVES = ROPE ? 2 : 1;
  __shared__ float2 angle[ROPE ? kAngles : 1];
  __shared__ int64_t to[kAppendRows];  // where a row's keys and values go, less the head; -1: nowhere, -2: the row is unused
  const int t0 = blockIdx.x * rows, here = min(rows, T - t0), tid = threadIdx.x;
  const int width = dh / HALVES, per_head = width / N, per_row = Hs * per_head, total = here * per_row;
  const int64_t HD = (int64_t)Hs * dh;
  E x[3][HALVES];
  int r = 0, h = 0, f = 0;
  auto load = [&](int i) {
    r = i / per_row;
    h = (i - r * per_row) / per_head;
    f = (i - r * per_row - h * per_head) * N;
    const int64_t in = (t0 + r) * ld + (int64_t)h * dh + f;
#pragma unroll
    for (int c = 0; c < 3; ++c)
#pragma unroll
      for (int a = 0; a < HALVES; ++a) x[c][a].load(qkv, in + c * HD + a * width);
  };
  int i = tid;
  if (i < total) load(i);
  if (const int row = tid - (kT - 64); row >= 0 && row < here) {  // (the last wave, which has no angles where rows are few: two chains of loads at once)
    const int p = max(0, lens[t0 + row]) - 1, s = seq ? seq[t0 + row] : t0 + row;
    int64_t at = -2;
    if (p >= 0 && (unsigned)s < (unsigned)pg.n_seqs) at = place(pg, page_stride, s, p, 0, dh);
    to[row] = at;
  }
  if (ROPE) {
    for (int j = tid; j < here * width; j += kT) {
      const int row = j / width, pair = j - row * width;
      rotation(max(1, lens[t0 + row]) - 1, turns.of(pair), angle[j].x, angle[j].y);
    }
  }
  __syncthreads();
  for (; i < total; ) {
    const int64_t at = to[r];
    if (at != -2) {
      if (ROPE) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float lo[N], hi[N];
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float2 w = angle[r * width + f + e];
            const float a = x[c][0].get(e), b = x[c][HALVES - 1].get(e);
            lo[e] = a * w.x - b * w.y;
            hi[e] = b * w.x + a * w.y;
          }
          x[c][0].set(lo);
          x[c][HALVES - 1].set(hi);
        }
      }
#pragma unroll
      for (int a = 0; a < HALVES; ++a) {
        if (q_out) x[0][a].store(q_out, (t0 + r) * ldq + (int64_t)h * dh + f + a * width);
        if (at >= 0) {
          const int64_t out = at + (((int64_t)h << pg.shift) * dh) + f + a * width;
          x[1][a].store(k, out);
          x[2][a].store(v, out);
        }
      }
    }
    i += kT;
    if (i < total) load(i);
  }
}

// ------------------------------------------------------------------------------------------- attention
constexpr int kMaxHead = 256;
constexpr int kMaxIds = 2048;    // pages that a part of a sequence lies on (their offsets are kept in LDS)
constexpr int kMaxParts = 1024;  // parts of a sequence

typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

// value of a lane from the lane that its row of 16 (or quad) permutation names
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// sum over aligned groups of G lanes, in every lane of the group
template <int G> __device__ __forceinline__ float group_sum(float v) {
  if (G > 1) v += dpp<0xB1>(v);    // quad_perm 1 0 3 2
  if (G > 2) v += dpp<0x4E>(v);    // quad_perm 2 3 0 1
  if (G > 4) v += dpp<0x141>(v);   // row_half_mirror: the other quad of 8
  if (G > 8) v += dpp<0x140>(v);   // row_mirror: the other 8 of 16
  if (G > 16) v += __shfl_xor(v, 16, 64);
  if (G > 32) v += __shfl_xor(v, 32, 64);
  return v;
}

// 16 bytes of a row of dh elements from element e on; element by element where rows are not aligned (zeros beyond the row)
template <int BF, bool VEC> __device__ __forceinline__ u32x4v piece(const void *p, int64_t i, int e, int dh) {
  constexpr int N = BF ? 8 : 4;
  if (VEC) return *reinterpret_cast<const u32x4v *>(static_cast<const char *>(p) + (i + e) * (16 / N));
  u32x4v r = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (e + j < dh) {
      if (BF) r[j / 2] |= (uint32_t) static_cast<const uint16_t *>(p)[i + e + j] << (16 * (j & 1));
      else r[j] = static_cast<const uint32_t *>(p)[i + e + j];
    }
  }
  return r;
}
template <int BF> __device__ __forceinline__ float value(const u32x4v &r, int j) {
  if (BF) return __uint_as_float(j & 1 ? r[j / 2] & 0xffff0000u : r[j / 2] << 16);
  return __uint_as_float(r[j]);
}

struct AttentionArgs {
  Pages pg;
  const void *k, *v, *q;
  int64_t page_stride, ldq, ldo;
  const int32_t *seq, *lens;
  void *o;
  float *lse, *acc_parts, *ml_parts;
  int32_t T, Hs, dh, max_len, parts, chunk;  // a sequence is cut into `parts` parts of `chunk` tokens
  int32_t turns, run, places;                // places: workgroups of a part; turns, run: how they are dealt out (see the kernels)
  float scale;
};

// the end of a row: o = acc / l, and lse; `seen`: it saw a token (if only with scores of -infinity, there is no number to give)
template <int BF> __device__ __forceinline__ void finish(const AttentionArgs &A, int t, int h, int e, float acc, float m, float l, bool seen) {
  store1<BF>(A.o, t * A.ldo + (int64_t)h * A.dh + e, seen ? acc / l : 0.f);
  if (e == 0 && A.lse) A.lse[(int64_t)t * A.Hs + h] = m == -INFINITY && l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718056f;
}

// what a workgroup found of a row of unit `unit`: the result, or a part of it
template <int BF> __device__ __forceinline__ void leave(const AttentionArgs &A, int64_t unit, int part, int t, int h, int e, float acc, float m, float l, bool seen) {
  if (A.parts == 1) {
    finish<BF>(A, t, h, e, acc, m, l, seen);
  } else {
    const int64_t at = unit * A.parts + part;
    A.acc_parts[at * A.dh + e] = acc;
    if (e == 0) reinterpret_cast<float2 *>(A.ml_parts)[at] = {m, seen && l == 0.f ? -1.f : l};  // (-1: tokens, but no weight)
  }
}

// Attention of one query to the keys of its sequence: with one key/value head per query head every key and value is used once, 4 flop for its 4 bytes (bf16),
// so reading them is the bound.  A workgroup of NW waves takes one (row, head, part).  G lanes hold a token, 16 bytes each, so a load instruction
// fetches 64 / G whole rows; a wave has four of them for keys and four for values in flight.  Every group of G lanes runs a softmax of its own over
// the tokens that it meets (running maximum and sum, one rescaling for four tokens), and nothing is exchanged until the end, where groups, waves
// and (in cache_attention_join_kernel) parts are joined by the usual rule.  Scores are in base 2: q carries scale * log2(e).
// Workgroups go to the 8 XCDs in turn, each with an L2 of its own: eight pairs of (run of A.run rows, head) with the runs' first rows, then the same
// eight with their next rows, so that rows of one sequence find what the first of them read (us for runs of 1 / 8: fp32, 13 heads of 256, 70 sequences of 91
// tokens, 5 rows each 78.7 / 39.9; 7 x 64, 24 of 1503, 3 rows 41.0 / 24.0; where heads are a multiple of 8 their rows are together anyway, 16 x 64, 8 of 100,
// 100 rows 24.5 / 27.8).
template <int BF, int G, bool VEC, int NW>
__global__ __launch_bounds__(64 * NW) void cache_attention_kernel(AttentionArgs A) {
  constexpr int N = BF ? 8 : 4, TPS = 64 / G, W = G * N, U = 4;
  __shared__ int64_t ids[kMaxIds];
  __shared__ float s_acc[NW][W], s_m[NW], s_l[NW];
  __shared__ int s_seen[NW];
  const int part = blockIdx.y, place = blockIdx.x;
  int pair = place, row = 0;
  if (A.run > 1) {
    pair = place / (8 * A.run) * 8 + place % 8;
    row = place / 8 % A.run;
  }
  const int h = pair % A.Hs, t = pair / A.Hs * A.run + row, unit = t * A.Hs + h;
  if (t >= A.T) return;
  const int s = A.seq ? A.seq[t] : t, given = A.lens[t], dh = A.dh;
  if (given < 0 || (unsigned)s >= (unsigned)A.pg.n_seqs) return;
  const int len = min(given, A.max_len), p0 = part * A.chunk, p1 = min(p0 + A.chunk, len);
  if (part && p0 >= len) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane / G, e = (lane % G) * N;
  const int shift = A.pg.shift, first = p0 >> shift, n_ids = p1 > p0 ? ((p1 - 1) >> shift) - first + 1 : 0;
  for (int i = tid; i < n_ids; i += 64 * NW) {
    const int page = A.pg.table[s * A.pg.ld + first + i];
    ids[i] = (unsigned)page < (unsigned)A.pg.n_pages ? page * A.page_stride + (((int64_t)h << shift)) * dh : -1;
  }
  float q[N], acc[N], m = -INFINITY, l = 0.f;
  const bool active = e < dh;
  const u32x4v qr = piece<BF, VEC>(A.q, t * A.ldq + (int64_t)h * dh, active ? e : 0, dh);
#pragma unroll
  for (int j = 0; j < N; ++j) { q[j] = active ? value<BF>(qr, j) * A.scale : 0.f; acc[j] = 0.f; }
  bool seen = false;
  __syncthreads();
  for (int tok0 = p0 + wave * (U * TPS); tok0 < p1; tok0 += NW * U * TPS) {
    u32x4v kr[U], vr[U];
    bool ok[U], all = true;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int tok = tok0 + u * TPS + g;
      const int64_t base = ids[min((tok >> shift) - first, n_ids - 1)];
      ok[u] = tok < p1 && base >= 0;
      all &= ok[u];
      const int64_t at = ok[u] ? base + (int64_t)(tok & ((1 << shift) - 1)) * dh : 0;  // (unused ones read the pool's first row)
      kr[u] = piece<BF, VEC>(A.k, at, active ? e : 0, dh);
      vr[u] = piece<BF, VEC>(A.v, at, active ? e : 0, dh);
    }
    __builtin_amdgcn_sched_barrier(0);  // (left alone, the compiler moves the values' loads behind the keys' use)
    float sc[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float d = 0.f;
#pragma unroll
      for (int j = 0; j < N; ++j) d = fmaf(q[j], value<BF>(kr[u], j), d);
      sc[u] = group_sum<G>(active ? d : 0.f);
    }
    if (!__all(all)) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        sc[u] = ok[u] ? sc[u] : -INFINITY;
        vr[u] = ok[u] ? vr[u] : u32x4v{0u, 0u, 0u, 0u};
        seen |= ok[u];
      }
    } else {
      seen = true;
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < U; ++u) mn = fmaxf(mn, sc[u]);
    const float ref = mn == -INFINITY ? 0.f : mn, c = __builtin_amdgcn_exp2f(m - ref);
    l *= c;
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] *= c;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float w = __builtin_amdgcn_exp2f(sc[u] - ref);
      l += w;
#pragma unroll
      for (int j = 0; j < N; ++j) acc[j] = fmaf(w, value<BF>(vr[u], j), acc[j]);
    }
    m = mn;
  }
  // the groups of the wave
#pragma unroll
  for (int off = G; off < 64; off *= 2) {
    const float m2 = __shfl_xor(m, off, 64), mn = fmaxf(m, m2), ref = mn == -INFINITY ? 0.f : mn;
    const float c = __builtin_amdgcn_exp2f(m - ref), c2 = __builtin_amdgcn_exp2f(m2 - ref);
    l = l * c + __shfl_xor(l, off, 64) * c2;
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = acc[j] * c + __shfl_xor(acc[j], off, 64) * c2;
    m = mn;
  }
  const bool wave_seen = __any(seen);
  if (lane < G) {
#pragma unroll
    for (int j = 0; j < N; ++j) s_acc[wave][e + j] = acc[j];
    if (lane == 0) { s_m[wave] = m; s_l[wave] = l; s_seen[wave] = wave_seen; }
  }
  __syncthreads();
  // the waves of the workgroup
  if (tid < dh) {
    float M = s_m[0];
    bool any = s_seen[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) { M = fmaxf(M, s_m[w]); any |= s_seen[w]; }
    const float ref = M == -INFINITY ? 0.f : M;
    float L = 0.f, a = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float c = __builtin_amdgcn_exp2f(s_m[w] - ref);
      L += c * s_l[w];
      a += c * s_acc[w][tid];
    }
    leave<BF>(A, unit, part, t, h, tid, a, M, L, any);
  }
}

// ------------------------------------------------------------------------------------------- rows that share a sequence
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef short s16x4v __attribute__((ext_vector_type(4)));
typedef short s16x8v __attribute__((ext_vector_type(8)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
constexpr int kTile = 16;  // rows of a tile

// Rows of the batch that follow each other and share a sequence (prompts, drafted tokens), up to RC tiles of kTile of them from a multiple of that on, read its
// keys once: a tile's scores are the 16 columns of v_mfma_f32_16x16x32_bf16.  S^T = K Q^T for two tiles of 16 tokens, the keys' fragments straight from memory: lane
// (j = lane / 16, c = lane % 16) holds 16 bytes of token c and gets the scores of tokens 4 j .. 4 j + 3 of either tile for row c.  These eight
// are the eight contraction indices that the lane has in O^T += V^T P^T, so the weights stay where they are; the values pass through LDS (a tile
// of the wave's own, no barrier) and come back transposed in the same order of tokens.  Weights go in as two bf16 terms, cut off and rounded: at most 2^-16 of
// them is lost, a fraction of the rounding of the output (2^-9).  What bounds it is the reading again, of 16 rows at once.
// fp32: v_mfma_f32_16x16x4_f32, of which an instruction takes one of the four numbers in a lane's 16 bytes of a key; four tokens of values are 4 x 256
// bytes as they lie, lane (j, c) with elements 4 c .. 4 c + 3 of token 4 j + e: number i of them belongs to an accumulator of elements 4 k + i, so that
// nothing passes through LDS.  Loads and products of a wave take turns: 45 to 60 % of the read rate, where one row a sequence reaches 75 to 93.
template <int BF, int KS, int NW, int RC>
__global__ __launch_bounds__(64 * NW) void cache_attention_tile_kernel(AttentionArgs A) {
  constexpr int ES = BF ? 2 : 4, N = 16 / ES, VB = (KS + 3) / 4, MT = BF ? 2 * KS : 4 * VB;
  constexpr int RB = 64 * KS + 32, LDR = 16 * MT + 4;  // bytes of a row of values in LDS, floats of one of results (the padding spreads the banks)
  constexpr int TILE_B = BF ? 32 * RB : kTile * LDR * 4;
  static_assert(kTile * LDR * 4 <= TILE_B, "results take the place of the values");
  __shared__ int64_t ids[kMaxIds];
  __shared__ __attribute__((aligned(16))) char tiles[NW][TILE_B];
  __shared__ float s_m[NW][kTile], s_l[NW][kTile];
  __shared__ int s_seen[NW][kTile];
  const int units = A.places / A.turns, unit = blockIdx.x % units, turn = blockIdx.x / units, part = blockIdx.y;
  const int h = unit % A.Hs, t0 = (RC > 1 ? units / A.Hs - 1 - unit / A.Hs : unit / A.Hs) * (RC * kTile), dh = A.dh;  // (a prompt's last rows, the longest, first)
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, j = lane >> 4, c = lane & 15;
  // the first rows of the groups among rows t0 .. t0 + 16 RC - 1, of which every A.turns-th is this workgroup's
  const bool mine = lane < RC * kTile && t0 + lane < A.T;
  const int own = mine ? A.seq[t0 + lane] : -1, prev = __shfl_up(own, 1, 64);
  uint32_t starts = (uint32_t)__ballot(mine && (lane == 0 || own != prev));
  for (int n = 0; starts; ++n) {
    const int r0 = __builtin_ctz(starts), t = t0 + r0;
    starts &= starts - 1;
    if (n % A.turns != turn) continue;
    const int rows = (starts ? __builtin_ctz(starts) : min(RC * kTile, A.T - t0)) - r0;
    const int s = __builtin_amdgcn_readfirstlane(__shfl(own, r0, 64));
    if ((unsigned)s >= (unsigned)A.pg.n_seqs) continue;
    int len[RC], top_len[RC], longest = -1, shortest = INT32_MAX;  // of the lane's row of each tile, of the tile
#pragma unroll
    for (int b = 0; b < RC; ++b) {
      const bool in = b * kTile + c < rows;
      len[b] = in ? min(A.lens[t + b * kTile + c], A.max_len) : -1;
      int hi = len[b], lo = in ? len[b] : INT32_MAX;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) {
        hi = max(hi, __shfl_xor(hi, o, 64));
        lo = min(lo, __shfl_xor(lo, o, 64));
      }
      top_len[b] = __builtin_amdgcn_readfirstlane(hi);
      longest = max(longest, top_len[b]);
      shortest = min(shortest, __builtin_amdgcn_readfirstlane(lo));
    }
    const int p0 = part * A.chunk, p1 = min(p0 + A.chunk, longest);
    if (longest < 0 || (part && p0 >= longest)) continue;
    const int shift = A.pg.shift, first = p0 >> shift, n_ids = p1 > p0 ? ((p1 - 1) >> shift) - first + 1 : 0;
    for (int i = tid; i < n_ids; i += 64 * NW) {
      const int page = A.pg.table[s * A.pg.ld + first + i];
      ids[i] = (unsigned)page < (unsigned)A.pg.n_pages ? page * A.page_stride + (((int64_t)h << shift)) * dh : -1;
    }
    const u32x4v none = {0u, 0u, 0u, 0u};
    u32x4v qf[RC][KS];
    f32x4v acc[RC][MT];
    float m[RC], l[RC];  // of the lane's row: the maximum of all scores, the sum of this lane's weights
    bool seen[RC];
#pragma unroll
    for (int b = 0; b < RC; ++b) {
      const char *q = static_cast<const char *>(A.q) + ((t + min(b * kTile + c, rows - 1)) * A.ldq + (int64_t)h * dh) * ES;
#pragma unroll
      for (int k = 0; k < KS; ++k) qf[b][k] = (4 * k + j) * N < dh ? *reinterpret_cast<const u32x4v *>(q + 64 * k + 16 * j) : none;
#pragma unroll
      for (int i = 0; i < MT; ++i) acc[b][i] = f32x4v{0.f, 0.f, 0.f, 0.f};
      m[b] = -INFINITY;
      l[b] = 0.f;
      seen[b] = false;
    }
    char *tile = tiles[wave];
    const int wr = c * RB + 16 * j, rd = (4 * j + (c >> 2)) * RB + (c & 3) * 8;  // where the lane's values go, and what it reads of 4 x 16 of them
    __syncthreads();
    for (int tok0 = p0 + 32 * wave; tok0 < p1; tok0 += 32 * NW) {
      u32x4v kf[2][KS], vf[2][BF ? KS : 4 * VB];
      uint32_t there = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int tok = tok0 + 16 * i + c;
        const int64_t base = ids[min((tok >> shift) - first, n_ids - 1)];
        const bool ok = tok < p1 && base >= 0;
        there |= ((uint32_t)__ballot(ok) & 0xffffu) << (16 * i);
        const int64_t at = (ok ? base + (int64_t)(tok & ((1 << shift) - 1)) * dh : 0) * ES + 16 * j;  // (unused ones read the pool's first row)
        const char *kp = static_cast<const char *>(A.k) + at, *vp = static_cast<const char *>(A.v) + at;
#pragma unroll
        for (int k = 0; k < KS; ++k) kf[i][k] = (4 * k + j) * N < dh ? *reinterpret_cast<const u32x4v *>(kp + 64 * k) : none;
        if constexpr (BF) {
#pragma unroll
          for (int k = 0; k < KS; ++k) vf[i][k] = (4 * k + j) * N < dh && ok ? *reinterpret_cast<const u32x4v *>(vp + 64 * k) : none;
        }
      }
      if constexpr (!BF) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tok = tok0 + 16 * i + 4 * j + e;
            const int64_t base = ids[min((tok >> shift) - first, n_ids - 1)];
            const bool ok = tok < p1 && base >= 0;
            const char *vp = static_cast<const char *>(A.v) + (ok ? base + (int64_t)(tok & ((1 << shift) - 1)) * dh : 0) * 4 + 16 * c;
#pragma unroll
            for (int k = 0; k < VB; ++k) vf[i][4 * k + e] = 64 * k + 4 * c < dh && ok ? *reinterpret_cast<const u32x4v *>(vp + 256 * k) : none;
          }
      }
      __builtin_amdgcn_sched_barrier(0);  // (all loads before the first product)
      float p[RC][8];
#pragma unroll
      for (int b = 0; b < RC; ++b) {
        if (RC > 1 && tok0 >= top_len[b]) {  // (rows of a prompt that end before these tokens)
#pragma unroll
          for (int e = 0; e < 8; ++e) p[b][e] = 0.f;
          continue;
        }
        f32x4v sc[2] = {f32x4v{0.f, 0.f, 0.f, 0.f}, f32x4v{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            if constexpr (BF) {
              sc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, kf[i][k]), __builtin_bit_cast(bf16x8v, qf[b][k]), sc[i], 0, 0, 0);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) sc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[i][k][e]), __uint_as_float(qf[b][k][e]), sc[i], 0, 0, 0);
            }
          }
        const bool whole = there == 0xffffffffu && tok0 + 32 <= shortest;
        uint32_t on = 0xffu;  // which of the lane's eight tokens its row sees
        if (!whole) {
          on = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int tok = 16 * (e >> 2) + 4 * j + (e & 3);
            if ((there >> tok & 1) && tok0 + tok < len[b]) on |= 1u << e;
            else sc[e >> 2][e & 3] = -INFINITY;
          }
        }
        seen[b] |= on != 0;
        float mx = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])), fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float mn = fmaxf(m[b], mx), ref = mn == -INFINITY ? 0.f : mn;
        if (__any(mn > m[b])) {
          const float alpha = __builtin_amdgcn_exp2f((m[b] - ref) * A.scale);
          l[b] *= alpha;
#pragma unroll
          for (int i = 0; i < MT; ++i) acc[b][i] *= alpha;
          m[b] = mn;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[b][e] = __builtin_amdgcn_exp2f((sc[e >> 2][e & 3] - ref) * A.scale);
          l[b] += p[b][e];
        }
      }
      if constexpr (BF) {
        u32x4v hi[RC], lo[RC];
#pragma unroll
        for (int b = 0; b < RC; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t x = __float_as_uint(p[b][2 * e]), y = __float_as_uint(p[b][2 * e + 1]);
            hi[b][e] = __builtin_amdgcn_perm(y, x, 0x07060302u);  // the upper halves
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            const f32x2 rest = {p[b][2 * e] - __uint_as_float(x & 0xffff0000u), p[b][2 * e + 1] - __uint_as_float(y & 0xffff0000u)};
            lo[b][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, bf16x2v));
          }
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        u16x2 top = {0, 0};  // largest magnitude among the values
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            *reinterpret_cast<u32x4v *>(tile + 16 * i * RB + wr + 64 * k) = vf[i][k];
#pragma unroll
            for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vf[i][k][e] & 0x7fff7fffu));
          }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // read by the wave's other lanes
        if (!__any(top.x >= 0x7f80 || top.y >= 0x7f80)) {
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            typedef s16x4v __attribute__((address_space(3))) * lds_ptr;
            const s16x4v x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(tile + rd + 32 * i)), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(tile + 16 * RB + rd + 32 * i));
            const bf16x8v vt = __builtin_bit_cast(bf16x8v, s16x8v{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]});
#pragma unroll
            for (int b = 0; b < RC; ++b) {
              if (RC > 1 && tok0 >= top_len[b]) continue;
              acc[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8v, hi[b]), acc[b][i], 0, 0, 0);
              acc[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8v, lo[b]), acc[b][i], 0, 0, 0);
            }
          }
        } else {  // infinities and NaNs, which times the zero of a term or of a hidden token are no number: one by one, for the rows that see them
#pragma unroll
          for (int b = 0; b < RC; ++b)
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll 1
              for (int x = 0; x < 4; ++x) {
                const int tok = 16 * (e >> 2) + 4 * x + (e & 3);
                const float w = __shfl(p[b][e], 16 * x + c, 64);
                if (!(there >> tok & 1) || tok0 + tok >= len[b]) continue;
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                  const u32x2v u = *reinterpret_cast<const u32x2v *>(tile + tok * RB + 32 * i + 8 * j);
                  acc[b][i][0] = fmaf(w, __uint_as_float(u.x << 16), acc[b][i][0]);
                  acc[b][i][1] = fmaf(w, __uint_as_float(u.x & 0xffff0000u), acc[b][i][1]);
                  acc[b][i][2] = fmaf(w, __uint_as_float(u.y << 16), acc[b][i][2]);
                  acc[b][i][3] = fmaf(w, __uint_as_float(u.y & 0xffff0000u), acc[b][i][3]);
                }
              }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the next tokens' values take the place of these
      } else {
        uint32_t top = 0;  // largest magnitude among the values
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int k = 0; k < 4 * VB; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = max(top, vf[i][k][e] & 0x7fffffffu);
        const bool finite = !__any(top >= 0x7f800000u);
#pragma unroll
        for (int b = 0; b < RC; ++b) {
          if (RC > 1 && tok0 >= top_len[b]) continue;
          if (finite) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
              for (int i = 0; i < MT; ++i)
                acc[b][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[e >> 2][(i & ~3) + (e & 3)][i & 3]), p[b][e], acc[b][i], 0, 0, 0);
          } else {  // as above; the values from memory again
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll 1
              for (int x = 0; x < 4; ++x) {
                const int tok = 16 * (e >> 2) + 4 * x + (e & 3);
                const float w = __shfl(p[b][e], 16 * x + c, 64);
                if (!(there >> tok & 1) || tok0 + tok >= len[b]) continue;
                const float *vp = static_cast<const float *>(A.v) + ids[((tok0 + tok) >> shift) - first] + (int64_t)((tok0 + tok) & ((1 << shift) - 1)) * dh;
#pragma unroll
                for (int k = 0; k < VB; ++k)
#pragma unroll
                  for (int r = 0; r < 4; ++r) {
                    const int el = 64 * k + 16 * j + 4 * r;
                    if (el < dh) {
                      const f32x4v u = *reinterpret_cast<const f32x4v *>(vp + el);
#pragma unroll
                      for (int i = 0; i < 4; ++i) acc[b][4 * k + i][r] = fmaf(w, u[i], acc[b][4 * k + i][r]);
                    }
                  }
              }
          }
        }
      }
    }
    float *res = reinterpret_cast<float *>(tile);
#pragma unroll
    for (int b = 0; b < RC; ++b) {
      if (RC > 1 && b * kTile >= rows) break;
      l[b] += __shfl_xor(l[b], 16, 64);
      l[b] += __shfl_xor(l[b], 32, 64);
      const uint64_t any = __ballot(seen[b]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if constexpr (BF) {
          *reinterpret_cast<f32x4v *>(res + c * LDR + 16 * i + 4 * j) = acc[b][i];
        } else {  // (elements 4 k + i % 4 of its 64)
          const int k = i >> 2, r = i & 3;
          *reinterpret_cast<f32x4v *>(res + c * LDR + 64 * k + 16 * j + 4 * r) = f32x4v{acc[b][4 * k][r], acc[b][4 * k + 1][r], acc[b][4 * k + 2][r], acc[b][4 * k + 3][r]};
        }
      }
      if (j == 0) { s_m[wave][c] = m[b]; s_l[wave][c] = l[b]; s_seen[wave][c] = (any >> c | any >> (c + 16) | any >> (c + 32) | any >> (c + 48)) & 1; }
      __syncthreads();
      for (int i = tid; i < min(rows - b * kTile, kTile) * dh; i += 64 * NW) {
        const int r = i / dh, e = i - r * dh, row = t + b * kTile + r, row_len = A.lens[row];
        if (row_len < 0 || (part && p0 >= min(row_len, A.max_len))) continue;
        float M = s_m[0][r];
        bool some = s_seen[0][r];
#pragma unroll
        for (int w = 1; w < NW; ++w) { M = fmaxf(M, s_m[w][r]); some |= s_seen[w][r]; }
        const float ref = M == -INFINITY ? 0.f : M;
        float L = 0.f, a = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const float x = __builtin_amdgcn_exp2f((s_m[w][r] - ref) * A.scale);
          L += x * s_l[w][r];
          a += x * reinterpret_cast<const float *>(tiles[w])[r * LDR + e];
        }
        leave<BF>(A, (int64_t)row * A.Hs + h, part, row, h, e, a, M * A.scale, L, some);
      }
      __syncthreads();
    }
  }
}

// Joins the parts of a (row, head): parts with m = maximum, l = sum of weights against it, acc likewise.  A thread takes an element of every
// (kT / D)-th part, D the power of two that holds a head, with its loads in flight together; the threads of an element are added in a fixed order.
template <int BF>
__global__ __launch_bounds__(kT) void cache_attention_join_kernel(AttentionArgs A, int dlog) {
  __shared__ float s_w[kMaxParts], s_l[kT / 64], s_m[kT / 64], s_a[kT];
  __shared__ int s_seen[kT / 64];
  const int unit = blockIdx.x, h = unit % A.Hs, t = unit / A.Hs, s = A.seq ? A.seq[t] : t, given = A.lens[t], tid = threadIdx.x;
  if (given < 0 || (unsigned)s >= (unsigned)A.pg.n_seqs) return;
  const int len = min(given, A.max_len), n = max(1, (len + A.chunk - 1) / A.chunk);
  const float2 *ml = reinterpret_cast<const float2 *>(A.ml_parts) + (int64_t)unit * A.parts;
  const float *parts = A.acc_parts + (int64_t)unit * A.parts * A.dh;
  float2 own[kMaxParts / kT];
  float M = -INFINITY;
#pragma unroll
  for (int j = 0; j < kMaxParts / kT; ++j) {
    const int i = tid + j * kT;
    own[j] = i < n ? ml[i] : float2{-INFINITY, 0.f};
    M = fmaxf(M, own[j].x);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  if ((tid & 63) == 0) s_m[tid >> 6] = M;
  __syncthreads();
  M = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  const float ref = M == -INFINITY ? 0.f : M;
  float L = 0.f;
  bool any = false;
#pragma unroll
  for (int j = 0; j < kMaxParts / kT; ++j) {
    const int i = tid + j * kT;
    const float w = __builtin_amdgcn_exp2f(own[j].x - ref);
    if (i < n) s_w[i] = w;
    L += w * own[j].y;
    any |= own[j].y != 0.f;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) L += __shfl_xor(L, o, 64);
  any = __any(any);
  if ((tid & 63) == 0) { s_l[tid >> 6] = L; s_seen[tid >> 6] = any; }
  __syncthreads();
  L = s_l[0] + s_l[1] + s_l[2] + s_l[3];
  any = s_seen[0] | s_seen[1] | s_seen[2] | s_seen[3];
  const int D = 1 << dlog, e = tid & (D - 1);
  float a = 0.f;
  if (e < A.dh) {
#pragma unroll 4
    for (int i = tid >> dlog; i < n; i += kT >> dlog) a += s_w[i] * parts[(int64_t)i * A.dh + e];
  }
  s_a[tid] = a;
  __syncthreads();
  if (tid >= A.dh) return;
  for (int i = 1; i < kT >> dlog; ++i) a += s_a[(i << dlog) + tid];
  finish<BF>(A, t, h, tid, a, M, L, any);
}

// Kernel, waves of a workgroup, parts of a sequence and their length, for T rows of Hs heads over at most max_len tokens.  n_seqs, the table's rows, stands for the
// sequences that the T rows are of (the host does not see whose they are; the caller may pass a table of those alone).  Figures are us on the device, launch included; heads of 128 in bf16 if nothing else is said, as (heads x sequences) x tokens.
//  - Tiles (turns > 0; a workgroup takes every turns-th group among 16 rows): where sequences have several rows each on average, the more the shorter they may be
//    (rows beyond 16 a sequence fill no more of a tile), and enough of both to fill the chip.  bf16, (heads x sequences) x tokens, r rows each, rows / tiles: (16 x 16) x 64, 16 rows 12.5 / 7.1,
//    (16 x 64) x 64, 8 rows 23.8 / 27.1, x 250 47 / 37.7, (12 x 32) of 64 x 100, 5 rows 8.8 / 10.9, x 300 15.8 / 15.6, (19 x 19) x 926, 8 rows 83 / 34.8, a prompt of 1024,
//    8 heads 172 / 34.5; few rows: (8 x 6) x 1172, 2 rows 12.6 / 17.3, (15 x 4) x 343, 8 rows 9.6 / 11.8, (30 x 2) of 64 x 1299, 8 rows 14.7 / 15.6.
//    fp32, whose matrix instruction has a sixteenth of the rate: (12 x 32) of 64 x 400, 5 rows 19.3 / 26, (16 x 16) of 64 x 128, 16 rows 13.5 / 9.6,
//    (29 x 24) of 96 x 1512, 8 rows 547 / 138, (12 x 8) of 64 x 1003, 4 rows 14.3 / 19, (16 x 4) x 4170, 3 rows 64 / 54, (12 x 40) of 64 x 2133, 2 rows 77 / 89; a prompt
//    of 2000, 16 heads 1168 / 343.
//    Two tiles in the registers of a workgroup, for heads that leave room for them (33 to 128), where sequences have 32 rows on average and many tokens.  One / two:
//    a prompt of 4096, 32 heads 1139 / 656, of 2000, 16 heads 174 / 112 (fp32 343 / 305), of 1024, 8 heads 34.5 / 30.4, of 512 17.2 / 23.2, 200 rows behind 7800, 8 heads 77.6 / 50.4, 4
//    prompts of 300 28.9 / 32.2; fp32, 12 heads of 64, 2 of 1000 90.7 / 77.1, 1 of 500 20.9 / 23.5; heads of 32, 16 x 2 of 1000 30.1 / 35.3, of 256, 4 x 2 67.6 / 74.9.
//  - Up to 384 KB of keys and values a head are read by one workgroup; where heads and rows are at most half the CUs, longer sequences are cut so that there are
//    256 of them, into parts of 64 KB at least (a second launch joins them, 4 us): uncut / that / finer: 12 heads of 64 x 1000 7.1 / - / 7.7, 8 x 1500 13 / 8.0 / -,
//    8 x 4096 22 / 10.5 / 11, 32 x 2048 17 / 12.6 / 12.5, 32 x 8192 - / 30.5 / 32.5, 16 x 32768 - / 53.4 / 55.2;
//    beyond that half, 12 heads of 64 x 16 in fp32 x 2000 32 / 35 / -.  Tiles, whose waves take 32 tokens at a time: 256 KB (16 heads x 4096, 8 rows: parts of 256 / 512 / 1024 22.9 / 18.5 / 25).
//  - Where workgroups are few enough that the longest row of all decides, parts of 1 MB even out rows of different lengths.  Rows, from 2.5 MB on, up to 1024 workgroups: uncut / cut (8 x 20) x
//    6000 82.5 / 76.5, x 8000 107 / 90, (12 x 16) x 6000 89.7 / 82.4, (16 x 32) x 6000 196 / 189, (32 x 16) x 16384 493 / 478, (16 x 64) x 8192 495 / 481, (8 x 32) x 6000 107 / 108.5;
//    on the other side (8 x 32) x 4096 74.7 / 79.3, (12 x 16) x 4096 60.6 / 65.7, (16 x 128) x 2048 238 / 246, x 6000 685 / 690, (32 x 128) x 6000 1351 / 1353.  Tiles, from 2 MB on, between 128
//    (below, what is said above) and 512: (7 x 20) x 12000, 2 rows 187 / 131, (5 x 36) x 9059, 5 rows 147 / 143, (8 x 36) 260 / 225, (20 x 8) x 8192, 8 rows 133 / 103,
//    (40 x 8) 208 / 194, but (16 x 16) x 6000, 16 rows 117 / 129; on the other side (16 x 8) x 8192, 8 rows 83 / 92, (16 x 32) 277 / 286, (32 x 64) x 6000, 4 rows 703 / 747.  Prompts (32 rows a
//    sequence and more), whose longest rows start first, are never cut for it: 4096 tokens, 32 heads 655 / 904, 8 heads 172 / 235, 8192, 2 heads 150 / 230, 1000 behind 6000, 8
//    heads 118 / 162, fp32 64 wide 176 / 205, bf16 4 heads of 256 217 / 311, 2000 behind 14000, 2 heads of 32 70 / 70.
//  - A workgroup of 16 waves draws 84 GB/s, one of 4 waves 42; 256 of either draw what the HBM gives.  Parts that cannot feed 16 waves take 4.  16 / 4 waves: 4
//    heads of 64 x 20 4.6 / 3.8, 12 x 1000 7.1 / 8.1, parts of 128 tokens 8.2 / 8.0, of 512 13.2 / 16.8; (16 x 128) x 200 39 / 29, (16 x 64) x 1000 62 / 64.  Tiles have 8
//    waves (what registers allow), or 4 where parts are short and workgroups more than CUs, 8 / 4: (16 x 64) x 250, 8 rows 37.5 / 29.2, (19 x 19) x 926, 8 rows 35.5 / 32.7,
//    (21 x 18) x 933, 2 rows 37.8 / 33.6, (16 x 8) of 64, prompts of 100 21.3 / 13.1; (16 x 8) x 1000, 16 rows 21.3 / 24.9, (30 x 10) x 1800, 8 rows 50 / 55.5; fp32 (16 x 64) x
//    300, 8 rows 70.5 / 78.9.
struct Split { int waves, parts, chunk, tiles, turns, run, places; };
Split choose_split(int T, int n_seqs, int Hs, int max_len, int shift, int dh, int es, bool listed, bool tiles) {
  Split s;
  const int64_t row_bytes = dh * es, pair = 2 * row_bytes;
  tiles = tiles && T >= (es == 2 ? 2 : 3) * (int64_t)n_seqs && std::min<int64_t>(16 * (int64_t)n_seqs, T) * max_len >= (es == 2 ? 1024 : 2048) * (int64_t)n_seqs &&
          (T * Hs >= 2048 || (int64_t)T * Hs * dh >= ((1 << 25) + max_len - 1) / max_len);
  s.tiles = tiles ? T >= 32 * (int64_t)n_seqs && max_len >= 768 && dh > 32 && dh <= 128 ? 2 : 1 : 0;
  const int rows = kTile * std::max(1, s.tiles);
  const int64_t blocks = (T + rows - 1) / rows;
  s.turns = tiles ? std::min({8, T, (int)(((int64_t)rows * n_seqs + T - 1) / T)}) : 0;
  s.run = listed && T >= 2 * (int64_t)n_seqs && Hs % 8 ? std::min(T, 8) : 1;
  s.places = (int)(tiles ? blocks * s.turns * Hs : s.run > 1 ? ((int64_t)(T + s.run - 1) / s.run * Hs + 7) / 8 * 8 * s.run : (int64_t)T * Hs);
  const int64_t units = (s.turns ? std::min(blocks * s.turns, n_seqs + blocks - 1) : T) * Hs;
  int64_t c = max_len;
  if (units <= 128 && max_len * pair > 384 << 10) c = std::max<int64_t>((s.turns ? 256 << 10 : 64 << 10) / pair, max_len / (256 / units));
  const bool even_out = s.turns ? max_len * pair >= 2048 << 10 && units > 128 && units < 512 && T < 32 * (int64_t)n_seqs : max_len * pair >= 2560 << 10 && units <= 1024;
  if (even_out) c = std::min<int64_t>(c, (1 << 20) / pair);
  c = std::max<int64_t>(c, (max_len + kMaxParts - 1) / kMaxParts);
  c = std::min<int64_t>((c + 63) / 64 * 64, (int64_t)(kMaxIds - 1) << shift);  // (one page more where it begins inside one)
  if (tiles) s.waves = es == 2 && units > 256 && c * row_bytes <= 256 << 10 ? 4 : 8;
  else s.waves = c * row_bytes > (units <= 256 ? 32 << 10 : 128 << 10) ? 16 : 4;
  s.chunk = (int)c;
  s.parts = (int)((max_len + c - 1) / c);
  return s;
}

twist_status check_pages(twist_ctx *ctx, const char *who, const twist_pages *p) {
  if (!p || !p->table) TW_FAIL(ctx, TWIST_EINVAL, "%s: null page table", who);
  if (p->n_seqs < 1 || p->max_pages < 1 || p->n_pages < 1) TW_FAIL(ctx, TWIST_EINVAL, "%s: a cache has at least one sequence and one page", who);
  if (p->ld_table < p->max_pages) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of the page table overlap", who);
  if (p->page_tokens < 1 || p->page_tokens > 4096 || (p->page_tokens & (p->page_tokens - 1)))
    TW_FAIL(ctx, TWIST_ESHAPE, "%s: page_tokens=%d is not a power of two up to 4096", who, p->page_tokens);
  if ((int64_t)p->max_pages * p->page_tokens > (int64_t)1 << 30) TW_FAIL(ctx, TWIST_ESHAPE, "%s: a sequence has room for 2^30 tokens at most", who);
  return TWIST_OK;
}

// the arguments that both calls have
twist_status check_cache(twist_ctx *ctx, const char *who, const twist_pages *p, int64_t page_stride, int T, int Hs) {
  TW_TRY(check_pages(ctx, who, p));
  const int64_t dh = ctx->d.d_head;
  if (T < 1 || Hs < 1) TW_FAIL(ctx, TWIST_EINVAL, "%s: empty input", who);
  if (dh > kMaxHead) TW_FAIL(ctx, TWIST_ESHAPE, "%s: d_head=%lld above %d is not supported", who, (long long)dh, kMaxHead);
  if ((int64_t)T * Hs >= (int64_t)1 << 22) TW_FAIL(ctx, TWIST_ESHAPE, "%s: %d rows of %d heads are too many for one call", who, T, Hs);
  if (page_stride < Hs * dh * p->page_tokens) TW_FAIL(ctx, TWIST_ESHAPE, "%s: page_stride=%lld is less than a page", who, (long long)page_stride);
  if (page_stride > INT64_MAX / 8 / p->n_pages) TW_FAIL(ctx, TWIST_ESHAPE, "%s: page_stride=%lld is beyond any memory", who, (long long)page_stride);
  return TWIST_OK;
}

Pages device_pages(const twist_pages *p) {
  return {p->table, p->ld_table, p->n_seqs, p->max_pages, p->n_pages, __builtin_ctz((unsigned)p->page_tokens)};
}

// listed: the rows' sequences are given (several may name one); vec: pieces of 16 bytes all through
Split attention_split(const twist_ctx *ctx, const twist_pages *p, int T, int Hs, int &max_len, bool listed, bool vec) {
  max_len = (int)std::min<int64_t>(max_len, (int64_t)p->max_pages * p->page_tokens);
  return choose_split(T, p->n_seqs, Hs, max_len, __builtin_ctz((unsigned)p->page_tokens), ctx->d.d_head, ctx->esize(), listed, listed && vec);
}
// whether it can be launched: workgroups of up to 1024 threads, of which a launch has less than 2^32, and parts that can be joined
bool launchable(const Split &s) { return s.parts <= kMaxParts && (int64_t)s.places * s.parts < (int64_t)1 << 22; }

void launch_attention_join(int bf16, hipStream_t st, const AttentionArgs &a) {
  int dlog = 0;
  while (1 << dlog < a.dh) ++dlog;
  if (bf16) hipLaunchKernelGGL((cache_attention_join_kernel<1>), dim3((unsigned)(a.T * a.Hs)), dim3(kT), 0, st, a, dlog);
  else hipLaunchKernelGGL((cache_attention_join_kernel<0>), dim3((unsigned)(a.T * a.Hs)), dim3(kT), 0, st, a, dlog);
}
template <int BF, int G, bool VEC>
void launch_attention(hipStream_t st, const AttentionArgs &a, int waves) {
  const dim3 grid((unsigned)a.places, (unsigned)a.parts);
  if (waves == 16) hipLaunchKernelGGL((cache_attention_kernel<BF, G, VEC, 16>), grid, dim3(1024), 0, st, a);
  else hipLaunchKernelGGL((cache_attention_kernel<BF, G, VEC, 4>), grid, dim3(256), 0, st, a);
}
template <int BF, bool VEC>
void launch_attention_of(hipStream_t st, const AttentionArgs &a, int waves) {
  const int pieces = (a.dh + (BF ? 7 : 3)) / (BF ? 8 : 4);
  if (pieces <= 1) launch_attention<BF, 1, VEC>(st, a, waves);
  else if (pieces <= 2) launch_attention<BF, 2, VEC>(st, a, waves);
  else if (pieces <= 4) launch_attention<BF, 4, VEC>(st, a, waves);
  else if (pieces <= 8) launch_attention<BF, 8, VEC>(st, a, waves);
  else if (pieces <= 16) launch_attention<BF, 16, VEC>(st, a, waves);
  else if (pieces <= 32) launch_attention<BF, 32, VEC>(st, a, waves);
  else if constexpr (!BF) launch_attention<BF, 64, VEC>(st, a, waves);
  if (a.parts > 1) launch_attention_join(BF, st, a);
}

template <int BF, int KS>
void launch_attention_tile_of(hipStream_t st, const AttentionArgs &a, const Split &split) {
  constexpr int NW = KS > (BF ? 4 : 8) ? 4 : 8, NW2 = KS > 4 ? 4 : 8;  // (what their registers allow)
  const dim3 grid((unsigned)a.places, (unsigned)a.parts);
  if constexpr (BF ? KS > 1 && KS <= 4 : KS > 2 && KS <= 8) {
    if (split.tiles == 2) {
      hipLaunchKernelGGL((cache_attention_tile_kernel<BF, KS, NW2, 2>), grid, dim3(64 * NW2), 0, st, a);
      return;
    }
  }
  if constexpr (BF && NW == 8) {
    if (split.waves == 4) {
      hipLaunchKernelGGL((cache_attention_tile_kernel<BF, KS, 4, 1>), grid, dim3(256), 0, st, a);
      return;
    }
  }
  hipLaunchKernelGGL((cache_attention_tile_kernel<BF, KS, NW, 1>), grid, dim3(64 * NW), 0, st, a);
}
void launch_attention_tile(int bf16, hipStream_t st, const AttentionArgs &a, const Split &split) {
  const int pieces = (a.dh * (bf16 ? 2 : 4) + 63) / 64;  // of 64 bytes
  if (bf16) {
    switch (pieces) {
      case 1: launch_attention_tile_of<1, 1>(st, a, split); break;
      case 2: launch_attention_tile_of<1, 2>(st, a, split); break;
      case 3: launch_attention_tile_of<1, 3>(st, a, split); break;
      case 4: launch_attention_tile_of<1, 4>(st, a, split); break;
      case 5: launch_attention_tile_of<1, 5>(st, a, split); break;
      case 6: launch_attention_tile_of<1, 6>(st, a, split); break;
      case 7: launch_attention_tile_of<1, 7>(st, a, split); break;
      default: launch_attention_tile_of<1, 8>(st, a, split); break;
    }
  } else if (pieces <= 2) {
    launch_attention_tile_of<0, 2>(st, a, split);
  } else if (pieces <= 4) {
    launch_attention_tile_of<0, 4>(st, a, split);
  } else if (pieces <= 8) {
    launch_attention_tile_of<0, 8>(st, a, split);
  } else if (pieces <= 12) {
    launch_attention_tile_of<0, 12>(st, a, split);
  } else {
    launch_attention_tile_of<0, 16>(st, a, split);
  }
  if (a.parts > 1) launch_attention_join(bf16, st, a);
}

bool al16(const void *p, int64_t stride_bytes = 0) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride_bytes % 16 == 0; }

}  // namespace

extern "C" twist_status twist_cache_append_raw(twist_ctx *ctx, const twist_pages *pages, void *k, void *v, int64_t page_stride, const void *qkv, int64_t ld,
                                               int32_t T, int32_t Hs, const int32_t *seq, const int32_t *lens, void *q_out, int64_t ldq) {
  const char *who = "twist_cache_append_raw";
  if (!ctx || !k || !v || !qkv || !lens) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  TW_TRY(check_cache(ctx, who, pages, page_stride, T, Hs));
  const int dh = ctx->d.d_head;
  const int64_t HD = (int64_t)Hs * dh;
  if (ld < 3 * HD || (q_out && ldq < HD)) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows overlap", who);
  const int rope = ctx->d.use_rope, es = ctx->esize(), width = rope ? dh / 2 : dh;
  Turns turns;
  std::copy(ctx->rope_turns, ctx->rope_turns + 8, turns.coarse);
  std::copy(ctx->rope_turns + 8, ctx->rope_turns + 24, turns.fine);
  // the widest pieces that a head's halves, and all addresses, are multiples of
  uintptr_t bits = reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(qkv) | (uintptr_t)(width * es) | (uintptr_t)(ld * es) |
                   (uintptr_t)(page_stride * es);
  if (q_out) bits |= reinterpret_cast<uintptr_t>(q_out) | (uintptr_t)(ldq * es);
  const int bytes = bits % 16 == 0 ? 16 : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 2;
  // rows of a workgroup: what keeps its threads busy, but 512 workgroups before that
  const int per_row = (int)(HD / (rope ? 2 : 1) * es / bytes);
  const int rows = std::max(1, std::min({kT / per_row, (T + 511) / 512, kAppendRows, rope ? kAngles / width : kAppendRows}));
  const dim3 grid((unsigned)((T + rows - 1) / rows));
#define APPEND(BF, BYTES)                                                                                                                                    \
  if (rope) hipLaunchKernelGGL((append_kernel<BF, BYTES, true>), grid, dim3(kT), 0, ctx->stream, device_pages(pages), k, v, page_stride, qkv, ld, T, Hs, dh, seq, \
                               lens, q_out, ldq, turns, rows);                                                                                               \
  else hipLaunchKernelGGL((append_kernel<BF, BYTES, false>), grid, dim3(kT), 0, ctx->stream, device_pages(pages), k, v, page_stride, qkv, ld, T, Hs, dh, seq,     \
                          lens, q_out, ldq, turns, rows)
  if (ctx->d.dtype == TWIST_BF16) {
    if (bytes == 16) { APPEND(1, 16); } else if (bytes == 8) { APPEND(1, 8); } else if (bytes == 4) { APPEND(1, 4); } else { APPEND(1, 2); }
  } else {
    if (bytes == 16) { APPEND(0, 16); } else if (bytes == 8) { APPEND(0, 8); } else { APPEND(0, 4); }
  }
#undef APPEND
  TW_HIP(ctx, hipGetLastError());
  return TWIST_OK;
}

extern "C" twist_status twist_cache_attention_floats(twist_ctx *ctx, const twist_pages *pages, int32_t T, int32_t Hs, int32_t max_len, size_t *floats) {
  const char *who = "twist_cache_attention_floats";
  if (!ctx || !floats) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  TW_TRY(check_pages(ctx, who, pages));
  TW_TRY(check_cache(ctx, who, pages, (int64_t)Hs * ctx->d.d_head * pages->page_tokens, T, Hs));
  if (max_len < 1) TW_FAIL(ctx, TWIST_EINVAL, "%s: max_len=%d", who, max_len);
  size_t need = 0;
  bool any = false;
  for (int form = 0; form < 3; ++form) {  // whether the caller's rows may share sequences, and how they are aligned, is not known here: the most of what can run
    int most = max_len;
    const Split s = attention_split(ctx, pages, T, Hs, most, form > 0, form > 1 && ctx->d.d_head * ctx->esize() % 16 == 0);
    if (!launchable(s)) continue;
    any = true;
    if (s.parts > 1) need = std::max(need, (size_t)T * Hs * s.parts * (ctx->d.d_head + 2));
  }
  if (!any) TW_FAIL(ctx, TWIST_ESHAPE, "%s: %d rows of %d heads over %d tokens are too many for one call", who, T, Hs, max_len);
  *floats = need;
  return TWIST_OK;
}

twist_status twist_cache_attention_check(twist_ctx *ctx, const char *who, const twist_pages *pages, int T, int Hs, int max_len, bool listed) {
  int most = max_len;
  if (!launchable(attention_split(ctx, pages, T, Hs, most, listed, ctx->d.d_head * ctx->esize() % 16 == 0)))
    TW_FAIL(ctx, TWIST_ESHAPE, "%s: %d rows of %d heads over %d tokens are too many for one call", who, T, Hs, max_len);
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
  if (reinterpret_cast<uintptr_t>(scratch) % 16) TW_FAIL(ctx, TWIST_ESHAPE, "%s: scratch must be 16-byte aligned", who);
  if (scratch_floats < need) TW_FAIL(ctx, TWIST_ESHAPE, "%s: scratch of %zu floats is smaller than the %zu needed", who, scratch_floats, need);
  const int dh = ctx->d.d_head;
  const int64_t HD = (int64_t)Hs * dh;
  if (ldq < HD || ldo < HD) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows overlap", who);
  AttentionArgs a{};
  a.pg = device_pages(pages);
  a.k = k; a.v = v; a.q = q; a.o = o;
  a.page_stride = page_stride; a.ldq = ldq; a.ldo = ldo;
  a.seq = seq; a.lens = lens; a.lse = lse;
  a.T = T; a.Hs = Hs; a.dh = dh; a.max_len = max_len;
  const int es = ctx->esize();
  const bool vec = dh * es % 16 == 0 && al16(k, page_stride * es) && al16(v) && al16(q, ldq * es);
  const Split split = attention_split(ctx, pages, T, Hs, a.max_len, seq != nullptr, vec);
  if (!launchable(split)) TW_FAIL(ctx, TWIST_ESHAPE, "%s: %d rows of %d heads over %d tokens are too many for one call", who, T, Hs, max_len);
  a.turns = split.turns; a.run = split.run; a.places = split.places; a.parts = split.parts; a.chunk = split.chunk;
  a.ml_parts = scratch;
  a.acc_parts = need ? scratch + (size_t)T * Hs * a.parts * 2 : nullptr;
  a.scale = 1.44269504089f / sqrtf((float)dh);
  if (split.turns) {
    launch_attention_tile(ctx->d.dtype == TWIST_BF16, ctx->stream, a, split);
    TW_HIP(ctx, hipGetLastError());
    return TWIST_OK;
  }
  if (ctx->d.dtype == TWIST_BF16) { if (vec) launch_attention_of<1, true>(ctx->stream, a, split.waves); else launch_attention_of<1, false>(ctx->stream, a, split.waves); }
  else { if (vec) launch_attention_of<0, true>(ctx->stream, a, split.waves); else launch_attention_of<0, false>(ctx->stream, a, split.waves); }
  TW_HIP(ctx, hipGetLastError());
  return TWIST_OK;
}
