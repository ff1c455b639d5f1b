// What is taken from a row of logits: a token drawn from it, or its k largest.  A row's columns have one order, larger logits first and equal ones by column; everything here is a
// beginning of it.
#include <cstddef>

#include "bins.h"
#include "nn.h"
#include "row.h"

namespace {

constexpr int kTop = 1024;   // the longest list
constexpr int kList = 1536;  // columns that are put in order by comparing them with each other
constexpr int kBins = 1024;
constexpr int kFew = 256;    // bins of a workgroup's largest
constexpr int kColumnBits = 20;
constexpr int kTable = 512;
constexpr int kByBins = 64;  // longer lists are put in order by bins

// Unsigned numbers in the order of a row's columns: the logit's place in 32 bits, the column (turned over) below it.  Columns that hold no number count as -infinity, -0 is 0.
__device__ __forceinline__ uint64_t place(float v, int c) {
  const uint32_t b = __float_as_uint(v == v ? v + 0.f : -INFINITY);
  return (uint64_t)(b ^ (b >> 31 ? 0xffffffffu : 0x80000000u)) << kColumnBits | ((1u << kColumnBits) - 1 - (uint32_t)c);
}
__device__ __forceinline__ float value_of(uint64_t p) {
  const uint32_t k = (uint32_t)(p >> kColumnBits);
  return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int column_of(uint64_t p) { return (1 << kColumnBits) - 1 - (int)(p & ((1u << kColumnBits) - 1)); }

// 2^x in 64 bits for x <= 0 (below -200: 2^-200): 2^f, f of the fraction in -1/2 .. 1/2, by a Chebyshev polynomial of degree 10, 2^-51 off.
__device__ __forceinline__ double power2(double x, int bits) {
  x = fmax(x, -200.0);
  const double n = rint(x), f = x - n;
  double p = 7.074194562613105e-09;
  p = fma(p, f, 1.020869083593037e-07);
  p = fma(p, f, 1.3215432534254118e-06);
  p = fma(p, f, 1.5252657257186041e-05);
  p = fma(p, f, 0.00015403530463727982);
  p = fma(p, f, 0.0013333558230170627);
  p = fma(p, f, 0.009618129107587253);
  p = fma(p, f, 0.05550410866444768);
  p = fma(p, f, 0.24022650695910158);
  p = fma(p, f, 0.69314718055995);
  p = fma(p, f, 1.0);
  return ldexp(p, (int)n + bits);
}

// What a workgroup shares while it searches a row
template <int NT> struct Search {
  union alignas(16) {  // (read four counts at a time)
    unsigned long long amount[kBins];
    uint32_t count[kBins];
  } bins;
  unsigned long long list[kList];    // places that may be taken, in any order; then what the sorted ones weigh
  unsigned long long sorted[kList];
  static constexpr int kMarks = 2 * kList;
  __device__ __forceinline__ uint32_t *marks() { return reinterpret_cast<uint32_t *>(sorted); }  // pieces that hold columns for the list (before there are any in order)
  unsigned long long found[2], wave_sum[NT / 64];
  float most[NT / 64], least[NT / 64];
  double table[kTable];
  float part[NT / 64];
  float hi, lo;  // of list_of_many's list
  int n, marked;
};

static_assert(alignof(Search<256>) % sizeof(u32x4v) == 0 && offsetof(Search<256>, bins) % sizeof(u32x4v) == 0, "bins are read as vectors");

// A value that all lanes have, known to be one: what depends on it is a branch of all
__device__ __forceinline__ int uniform_of(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float uniform_of(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }
__device__ __forceinline__ unsigned long long uniform_of(unsigned long long v) {
  return (unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
}

template <int NT> __device__ __forceinline__ Search<NT> &shared() {
  __shared__ Search<NT> s;
  return s;
}

// A workgroup's steps over a row that it reads again for every pass: what is seldom needed, or takes long in any case.  Nothing here touches the row in registers.
template <int BF, int NT> struct Finder {
  using P16 = Piece<BF>;
  static constexpr int N = P16::N, NW = NT / 64;
  Search<NT> &sh;
  device_bytes row, first;
  int V, head, pieces, tid, wave, lane;

  __device__ __forceinline__ Finder(Search<NT> &s, device_bytes row_, int V_, int head_, int wave_) : sh(s), row(row_), V(V_), head(head_), tid(threadIdx.x), wave(wave_) {
    lane = tid & 63;
    pieces = (V - head) / N;
    first = row + head * P16::ES;
  }
  // f(N logits, the first's column, how many of them are the row's) for all of the row, with D pieces on their way: the registers of one that is done take the one D behind it
  // (not before it is done, and whether there is one or not: otherwise it is loaded somewhere else and waited for, to be moved)
  template <int D, class F> __device__ __forceinline__ void runs(F f) const {
    if (pieces > 0) {
      P16 next[D];
#pragma unroll
      for (int d = 0; d < D; ++d) next[d].load(first + (int64_t)min(tid + d * NT, pieces - 1) * 16);
#pragma unroll 1
      for (int v = tid; v < pieces; v += D * NT) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
          if (v + d * NT < pieces) {
            float x[N];
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = next[d][e];
            f(x, head + (v + d * NT) * N, N);
          }
          __builtin_amdgcn_sched_barrier(0);
          next[d].load(first + (int64_t)min(v + (d + D) * NT, pieces - 1) * 16);
        }
      }
    }
    const int c = tid < head ? tid : pieces * N + tid;
    if (tid < V - pieces * N) {
      float x[N];
      x[0] = load1<BF>(row, c);
#pragma unroll
      for (int e = 1; e < N; ++e) x[e] = -INFINITY;
      f(x, c, 1);
    }
  }
  // the number by which a run is marked
  __device__ __forceinline__ int piece_of(int c, int n) const { return n > 1 ? (c - head) / N : pieces + tid; }
  // f(logit, column) of every column.  SHORT: in one copy of f for each piece on its way instead of one for each of its logits, for functions of many passes.  A branch reaches
  // 128 KiB; in a function beyond that the compiler jumps through the registers of the return address, and the call does not return.
  template <bool SHORT = false, class F> __device__ __forceinline__ void columns(F f) const {
    if (SHORT)
      runs<2>([&](const float *x, int c, int n) {
#pragma unroll 1
        for (int e = 0; e < (n > 1 ? N : 1); ++e) {
          float v = x[0];
#pragma unroll
          for (int j = 1; j < N; ++j) v = e == j ? x[j] : v;
          f(v, c + e);
        }
      });
    else runs<4>([&](const float *x, int c, int n) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e == 0 || n > 1) f(x[e], c + e);
    });
  }
  __device__ __forceinline__ unsigned long long block_add(unsigned long long v) const {
    v = wave_add(v);
    __syncthreads();
    if (lane == 0) sh.wave_sum[wave] = v;
    __syncthreads();
    unsigned long long s = 0;
#pragma unroll 4
    for (int w = 0; w < NW; ++w) s += sh.wave_sum[w];
    return uniform_of(s);
  }
  template <class T> __device__ __forceinline__ void clear(T *bins, int n) const {
    for (int i = tid; i < n; i += NT) bins[i] = 0;
  }
  // The bin in which what lies in the bins up to it reaches `target` (n: none), and what lies before it.  n: 64 times a power of two.
  template <class T> __device__ __forceinline__ int find(const T *bins, int n, unsigned long long target, unsigned long long &before) const {
    if (wave == 0) {
      const int per = n / 64;
      unsigned long long s = 0, upto;
      for (int i = 0; i < per; ++i) s += bins[lane * per + ((i + lane) & (per - 1))];  // (in an order of its own: otherwise all lanes read from the same banks)
      upto = wave_sums(s);
      const uint64_t hit = __ballot(upto >= target);
      if (hit == 0) {
        if (lane == 63) { sh.found[0] = n; sh.found[1] = upto; }
      } else if (lane == __builtin_ctzll(hit)) {
        upto -= s;
        int b = lane * per;
        for (const int end = b + per - 1; b < end && upto + bins[b] < target; ++b) upto += bins[b];
        sh.found[0] = b;
        sh.found[1] = upto;
      }
    }
    __syncthreads();
    before = uniform_of(sh.found[1]);
    return uniform_of((int)sh.found[0]);
  }

  // The last place of the shortest beginning of the row whose columns' amounts add up to `target` (at least 1, at most the whole row's), a few bits of the places at a time.
  template <bool SHORT = false, class F> __device__ __forceinline__ uint64_t reach(unsigned long long target, F amount) const {
    uint64_t prefix = 0;
    int shift = 32 + kColumnBits;
#pragma unroll 1
    while (shift > 0) {
      const int w = shift > 12 ? 10 : 6, bins = 1 << w, above = shift;
      shift -= w;
      __syncthreads();
      clear(sh.bins.amount, bins);
      __syncthreads();
      columns<SHORT>([&](float v, int c) {
        const uint64_t p = place(v, c);
        if (p >> above != prefix) return;
        const unsigned long long a = amount(v, p);
        if (a) atomicAdd(&sh.bins.amount[bins - 1 - (int)(p >> shift & (bins - 1))], a);
      });
      __syncthreads();
      unsigned long long before;
      const int b = find(sh.bins.amount, bins, target, before);
      target -= before;
      prefix = prefix << w | (uint64_t)(bins - 1 - b);
    }
    __syncthreads();
    return prefix;
  }
  // the row's largest logit and the smallest above -infinity
  __device__ __forceinline__ void extremes(float &top, float &least) const {
    float m = -INFINITY, l = INFINITY;
    runs<6>([&](const float *x, int, int) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        m = fmaxf(m, x[e]);
        l = fminf(l, x[e] > -INFINITY ? x[e] : INFINITY);
      }
    });
    m = wave_max(m);
    l = -wave_max(-l);
    __syncthreads();
    if (lane == 0) { sh.most[wave] = m; sh.least[wave] = l; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) { m = fmaxf(m, sh.most[w]); l = fminf(l, sh.least[w]); }
    top = uniform_of(m);
    least = uniform_of(l);
  }
  // A logit that k columns at least are not below (none above -infinity is, where there are fewer), by counting all in bins.  -infinity: no bins for them.
  __device__ __forceinline__ float bound_of_all(int k, float &top) const {
    float l;
    extremes(top, l);
    const float span = top - l;
    if (!(top > -INFINITY) || !(span < INFINITY)) return -INFINITY;
    const float scale = bin_scale(kBins, span);
    clear(sh.bins.count, kBins);
    __syncthreads();
    columns([&](float v, int) {
      if (v > -INFINITY) atomicAdd(&sh.bins.count[(int)((top - v) * scale)], 1u);
    });
    __syncthreads();
    unsigned long long before;
    const int b = find(sh.bins.count, kBins, k, before);
    return b < kBins ? bin_edge(b, top, scale) : l;
  }
  // The list of the row's columns that are `wanted(logit, column)`, in two steps: pieces (and, behind their numbers, the columns in none) that hold one are marked in a pass over
  // the row, and looked through afterwards, a thread each.  A pass marks in few instructions; with what the list takes behind every column it is code that was not fetched before
  // (2.4 and 6.4 us where both steps take 1.8 and 2.9).  begin(); mark() in a pass; then take(), the columns' number, which may be more than the list holds.
  __device__ __forceinline__ void begin() const {
    __syncthreads();
    if (tid == 0) sh.n = sh.marked = 0;
    __syncthreads();
  }
  __device__ __forceinline__ void mark(int v) const {
    const int i = atomicAdd(&sh.marked, 1);
    if (i < Search<NT>::kMarks) sh.marks()[i] = v;
  }
  template <class F> __device__ __forceinline__ int take(F wanted) const {
    __syncthreads();
    const int n = uniform_of(sh.marked);
    if (n > Search<NT>::kMarks) return n;
#pragma unroll 1
    for (int i = tid; i < n; i += NT) {
      const int v = (int)sh.marks()[i], end = v - pieces;
      P16 y;
      y.u = P16::none();
      if (end < 0) y.load(first + (int64_t)v * 16);
      const int c = end < 0 ? head + v * N : end < head ? end : pieces * N + end;
      const float alone = end < 0 ? 0.f : load1<BF>(row, c);
#pragma unroll 1
      for (int e = 0; e < (end < 0 ? N : 1); ++e) {
        float x = alone;
#pragma unroll
        for (int j = 0; j < N; ++j) x = end < 0 && e == j ? y[j] : x;
        if (!wanted(x, c + e)) continue;
        const int at = atomicAdd(&sh.n, 1);
        if (at < kList) sh.list[at] = place(x, c + e);
      }
    }
    __syncthreads();
    return uniform_of(sh.n);
  }

  // What bound_of and the first list need, before the first barrier
  __device__ __forceinline__ void prepare() const {
    clear(sh.bins.count, kFew);
    if (tid == 0) sh.n = sh.marked = 0;
  }
  // Puts the list's n places in order, in sh.sorted: the first `most` of them.
  __device__ __forceinline__ void sort(int n, int most) const { sort(sh, tid, n, most); }
  static __device__ __forceinline__ void sort(Search<NT> &sh, int tid, int n, int most) {
    constexpr int U = 8;  // places that are read together
#pragma unroll 1
    for (int i = tid; i < n; i += NT) {
      const unsigned long long p = sh.list[i];
      int at = 0, j = 0;
#pragma unroll 1
      for (; j + U <= n; j += U)
#pragma unroll
        for (int u = 0; u < U; ++u) at += sh.list[j + u] > p;
#pragma unroll 1
      for (; j < n; ++j) at += sh.list[j] > p;
      if (at < most) sh.sorted[at] = p;
    }
    __syncthreads();
  }
  // The same of places from `hi` down to `lo` (not below it), all of them: counted in bins, put together by bin, and compared with those of their own bin alone.  Top 32, 64, 256
  // of 2048 x 32000 bf16: 42.8, 48.7 and 56.4 us, by comparing all with all 42.0, 51.0 and 72.9; top 512 of 2048 x 50257 104 and 166; 64 x 50257 fp32, top 64 and 1000, 11.7 and
  // 19.4 against 12.0 and 55.8.
  static __device__ __forceinline__ void sort_by_bins(Search<NT> &sh, int tid, int n, float hi, float scale) {
    uint32_t *bins = sh.bins.count;
    auto bin = [&](uint64_t p) { return min((int)((hi - value_of(p)) * scale), kFew - 1); };
    for (int i = tid; i < kFew; i += NT) bins[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += NT) atomicAdd(&bins[bin(sh.list[i])], 1u);
    __syncthreads();
    if (tid < 64) {
      u32x4v &own = *reinterpret_cast<u32x4v *>(bins + 4 * tid);
      const u32x4v c = own;
      const uint32_t sum = (c[0] + c[1]) + (c[2] + c[3]), before = wave_sums(sum) - sum;
      own = u32x4v{before, before + c[0], before + c[0] + c[1], before + c[0] + c[1] + c[2]};
    }
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
      const uint64_t p = sh.list[i];
      sh.sorted[atomicAdd(&bins[bin(p)], 1u)] = p;  // (afterwards a bin's number is where the next one begins)
    }
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < n; i += NT) {
      const uint64_t p = sh.sorted[i];
      const int b = bin(p), end = bins[b];
      const int start = b ? bins[b - 1] : 0;
      int at = start;
#pragma unroll 1
      for (int j = start; j < end; ++j) at += sh.sorted[j] > p;
      sh.list[at] = p;
    }
    __syncthreads();
    for (int i = tid; i < n; i += NT) sh.sorted[i] = sh.list[i];
    __syncthreads();
  }
};

// The row's largest logit (the thread's: `mine`), and the smallest of the threads' largest
template <int NT, class R> __device__ __forceinline__ void extremes(R &row, Search<NT> &sh, int wave, int lane, float &mine, float &top, float &low) {
  float m = fmaxf(row.xl, -INFINITY);
  row.each([&](const typename R::P16 &y, int) { m = fmaxf(m, y.most()); });
  mine = m;
  top = wave_max(m);
  low = -wave_max(m > -INFINITY ? -m : -INFINITY);
  if (lane == 0) { sh.most[wave] = top; sh.least[wave] = low; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) { top = fmaxf(top, sh.most[w]); low = fminf(low, sh.least[w]); }
  top = uniform_of(top);
  low = uniform_of(low);
}
// A logit that k columns at least are not below, and not many more where logits differ, by counting in bins the threads' largest or the pieces'.  -infinity: none was found, or k
// is above the workgroup's threads (the pieces would give a bound then too, with another `low`): such rows are read three times more, top 512 of 2048 x 32000 bf16 139 us where
// 256 take 58, drawing from the top 1000 of 4096 x 32000 499 where 50 take 72.
template <int BF, int NT, class R> __device__ __forceinline__ float bound_of(R &row, const Finder<BF, NT> &f, int k, float mine, float top, float low) {
  const float span = top - low;
  if (k > NT || !(top > -INFINITY) || !(span < INFINITY)) return -INFINITY;
  const float scale = bin_scale(kFew, span);
  auto put = [&](float v) {
    if (v >= low) atomicAdd(&f.sh.bins.count[(int)((top - v) * scale)], 1u);
  };
  if (8 * k <= NT) put(mine);
  else {
    row.each([&](const typename R::P16 &y, int) { put(y.most()); });
    put(row.xl);
  }
  __syncthreads();
  // every wave for itself: the bin in which the count reaches k
  const u32x4v own = *reinterpret_cast<const u32x4v *>(f.sh.bins.count + 4 * f.lane);
  const uint32_t sum = (own[0] + own[1]) + (own[2] + own[3]), upto = wave_sums(sum);
  const uint64_t hit = __ballot(upto >= (uint32_t)k);
  if (!hit) return -INFINITY;
  const int who = __builtin_ctzll(hit);
  uint32_t before = upto - sum;
  int b = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    before += own[i];
    b += before < (uint32_t)k;
  }
  return bin_edge(4 * who + __builtin_amdgcn_readlane(b, who), top, scale);
}
// the list from the columns at `from` and above; their number, which may be more than the list holds
template <int BF, int NT, class R> __device__ __forceinline__ int collect(R &row, const Finder<BF, NT> &f, float from) {
  row.each([&](const typename R::P16 &y, int v) {
    if (y.most() >= from) f.mark(v);
  });
  if (row.xl >= from) f.mark(row.pieces + f.tid);
  return f.take([&](float v, int) { return v >= from; });
}

// The list of a row's k first places (k at most its columns; in any order, and more where that is as quick), by counting all of its columns in bins, or else bit by bit; their
// number.  Every column of the list is before all others.  A function of its own, which leaves the registers of the quicker way alone.
template <int BF, int NT> __device__ __attribute__((noinline)) int list_of_many(device_bytes at_row, int V, int head, int wave, int k) {
  Search<NT> &sh = shared<NT>();
  const Finder<BF, NT> f(sh, at_row, V, head, wave);
  float top;
  const float from = f.bound_of_all(k, top);
  int n = 0;
  auto list = [&](float lo, auto wanted) {
    f.begin();
    if (f.tid == 0) { sh.hi = top; sh.lo = lo; }
    f.template runs<4>([&](const float *x, int c, int n) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < Piece<BF>::N; ++e) any |= (e == 0 || n > 1) && wanted(x[e], c + e);
      if (any) f.mark(f.piece_of(c, n));
    });
    return f.take(wanted);
  };
  if (from > -INFINITY) n = list(from, [&](float v, int) { return v >= from; });
  if (n < k || n > kList) {
    const uint64_t last = k < V ? f.reach(k, [](float, uint64_t) -> unsigned long long { return 1; }) : 0;
    n = list(last ? value_of(last) : -INFINITY, [&](float v, int c) { return place(v, c) >= last; });
  }
  return n;
}

// One row's settings and what follows from them: probabilities are whole multiples of 2^-bits of the largest, in 64 bits, so that any order of their sums gives the same.
struct Weigher {
  float top;
  double c;  // log2(e) / temperature
  int bits;
  __device__ __forceinline__ double exponent(float v) const { return v == top ? 0.0 : ((double)v - (double)top) * c; }  // of 2
  __device__ __forceinline__ double logarithm(float v, unsigned long long total) const { return exponent(v) * 0.6931471805599453 - log(ldexp((double)total, -bits)); }
  __device__ __forceinline__ unsigned long long operator()(float v) const {
    if (!(v > -INFINITY)) return 0;
    // (added to 2^52 the number is rounded to whole ones, which its last 52 bits are)
    return (unsigned long long)__double_as_longlong(power2(exponent(v), bits) + 4503599627370496.0) & 0xfffffffffffffull;
  }
  // The smallest logit whose probability is `least` of the largest: near where the logarithm says, a lane a value, otherwise by halving.
  __device__ float smallest(double least, int lane) const {
    if (least >= 1.0) return c > 0.0 || top == INFINITY ? top : -3.402823466e38f;  // (at an infinite temperature all are as probable)
    auto key = [](float v) { const uint32_t b = __float_as_uint(v); return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u); };
    auto value = [](uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); };
    auto enough = [&](uint32_t k) { return power2(exponent(value(k)), 0) >= least; };
    uint32_t lo = key(-3.402823466e38f), hi = key(top);
    const uint32_t guess = key((float)((double)top + log2(least) / c));
    if (guess > lo + 32 && guess < hi) {
      const uint64_t yes = __ballot(guess - 32 + lane >= hi || enough(guess - 32 + lane));
      if (yes && !(yes & 1)) return value(min(hi, guess - 32 + (uint32_t)__builtin_ctzll(yes)));
    }
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo) / 2;
      if (enough(mid)) hi = mid;
      else lo = mid + 1;
    }
    return value(lo);
  }
};

// The same for whole rows, in half the instructions (an exponential of power2 takes 25, several of which run at a fraction of the rate): 2^(n / 512) from a table, the rest of
// the exponent by a polynomial of degree 3 (2^-48 off).  Not for every row: `usable` tells.
struct QuickWeigher {
  double top, c;  // 512 log2(e) / temperature
  float least;    // below it nothing weighs anything
  const double *table;
  bool usable;
  __device__ __forceinline__ QuickWeigher(const Weigher &w, const double *t) : top(w.top), c(w.c * kTable), table(t) {
    least = fmaxf((float)(top - 190.0 / w.c), -3.402823466e38f);
    const double span = (top - (double)least) * w.c;  // (rounded to fp32 it may be anything, for instance where the temperature is next to nothing)
    usable = w.top < INFINITY && span <= 250.0 && (span >= 100.0 || least == -3.402823466e38f);
  }
  static __device__ __forceinline__ double entry(int i, int bits) { return power2((double)i / kTable - 1.0, bits + 1); }  // of the table
  __device__ __forceinline__ unsigned long long operator()(float v) const {
    const double d = (double)fmaxf(v, least) - top;
    const double m = fma(d, c, 6755399441055744.0), r = fma(d, c, -(m - 6755399441055744.0));  // (1.5 2^52: rounds to whole numbers, which the last bits are)
    const int n = __double2loint(m);
    double q = fma(r, 4.1353784691025013e-10, 9.163914342180769e-07);
    q = fma(q, r, 0.0013538030870311425);
    q = fma(q, r, 1.0) * table[n & (kTable - 1)];
    q = __hiloint2double(__double2hiint(q) + (n >> 9 << 20), __double2loint(q)) + 4503599627370496.0;
    return v > -INFINITY ? (unsigned long long)__double_as_longlong(q) & 0xfffffffffffffull : 0;
  }
};

// What wave 0 makes of n places in order (in LDS) that weigh weights[0 .. n): sums up to every one, 64 runs of them side by side.
struct Sums {
  const unsigned long long *weights;
  int n, per, lane;
  unsigned long long before, own, total;
  __device__ __forceinline__ Sums(const unsigned long long *w, int n_, int lane_) : weights(w), n(n_), lane(lane_) {
    per = (n + 63) / 64;
    own = 0;
    for (int i = lane * per; i < min(n, lane * per + per); ++i) own += weights[i];
    const unsigned long long upto = wave_sums(own);
    before = upto - own;
    total = last_of(upto);
  }
  // the first of them up to which they weigh `target`, and what they do (target at most the total)
  __device__ __forceinline__ int reach(unsigned long long target, unsigned long long &upto) const {
    const uint64_t hit = __ballot(before + own >= target);
    const int who = hit ? __builtin_ctzll(hit) : 63;
    unsigned long long s = before;
    int i = lane * per;
    if (lane == who)
      for (; i < n; ++i) {
        s += weights[i];
        if (s >= target) break;
      }
    upto = __shfl(s, who, 64);
    return __shfl(i, who, 64);
  }
  __device__ __forceinline__ unsigned long long upto(int count) const {  // what the first `count` weigh
    unsigned long long s = 0;
    for (int i = lane * per; i < min(count, min(n, lane * per + per)); ++i) s += weights[i];
    return wave_add(s);
  }
};

// One row's settings
struct Settings {
  float u, temp, p, m;
  int k;
  // the first sum that is `part` of the total or more
  static __device__ __forceinline__ unsigned long long share(double part, unsigned long long total) {
    const double s = ceil(part * (double)total);
    return s >= 1.0 ? min((unsigned long long)s, total) : 1ull;
  }
  __device__ __forceinline__ unsigned long long draw_at(unsigned long long total) const { return u > 0.f ? min((unsigned long long)((double)fminf(u, 1.f) * (double)total), total - 1) + 1 : 1ull; }
};

// A token of a row of which many columns may be kept: the probabilities of the whole row are added up in bins of their size, and the columns of the bin in which a sum (top_p's,
// the random number's) ends are put in order.  A function of its own, which leaves the registers of the way through a list alone.
template <int BF, int NT>
__device__ __attribute__((noinline)) void draw_of_many(device_bytes at_row, int V, int head, int wave, int bits, const Settings set, int32_t *token, float *logprob_out, int32_t *kept) {
  Search<NT> &sh = shared<NT>();
  const Finder<BF, NT> f(sh, at_row, V, head, wave);
  const int tid = f.tid, lane = f.lane, k = set.k;
  float top, lowest;
  f.extremes(top, lowest);
  if (!(top > -INFINITY)) {
    if (tid == 0) {
      *token = -1;
      if (logprob_out) *logprob_out = -INFINITY;
      if (kept) *kept = 0;
    }
    return;
  }
  const Weigher slow{top, 1.4426950408889634 / (double)set.temp, bits};
  for (int i = tid; i < kTable; i += NT) sh.table[i] = QuickWeigher::entry(i, bits);
  const QuickWeigher quick(slow, sh.table);
  const bool usable = uniform_of((int)quick.usable);
  const float p = set.p, m = set.m, least = m > 0.f ? uniform_of(slow.smallest(m, lane)) : -INFINITY;
  // the last place that is kept: of more than kTop columns bit by bit, in seven passes before the others (from the top 2000 of 64 x 32000 bf16: 68 us, of 64 x 50257 fp32 85)
  uint64_t last = 0;
  if (k > 1 && k < V) {
    unsigned long long n = 0;
    f.template columns<true>([&](float v, int) { n += v > -INFINITY; });
    if ((unsigned long long)k < f.block_add(n)) last = f.reach(k, [](float v, uint64_t) -> unsigned long long { return v > -INFINITY; });
  }
  auto mass = [&](float v) { return usable ? quick(v) : slow(v); };
  // min_p alone: its columns, where they are few, are all there is to weigh (64 x 32000 bf16, min_p 0.05: 32 us by bins, 13 so.  top_p's beginning is as a rule long: put in
  // order as a whole instead of the columns of one bin of it, 64 x 32000 with top_p 0.9 take 88 us instead of 32)
  if (m > 0.f && !(p < 1.f)) {
    f.begin();
    f.template runs<4>([&](const float *x, int c, int n) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < Piece<BF>::N; ++e) any |= x[e] >= least;
      if (any) f.mark(f.piece_of(c, n));
    });
    const int n = f.take([&](float v, int c) { return v >= least && place(v, c) >= last; });
    if (n <= kList) {
      f.sort(n, n);
      for (int i = tid; i < n; i += NT) sh.list[i] = mass(value_of(sh.sorted[i]));
      __syncthreads();
      if (wave) return;
      const Sums sums(sh.list, n, lane);
      unsigned long long upto;
      const int i = sums.reach(set.draw_at(sums.total), upto);
      if (lane == 0) {
        const uint64_t at = sh.sorted[i];
        *token = column_of(at);
        if (logprob_out) *logprob_out = (float)slow.logarithm(value_of(at), sums.total);
        if (kept) *kept = n;
      }
      return;
    }
  }
  // bins of equal width from the largest logit down to the smallest, or to where probabilities are below 2^-48
  const float span = fminf(top - lowest, 48.f * (float)(1.0 / slow.c)), scale = span < INFINITY ? bin_scale(kBins, span) : 0.f;
  auto bin = [&](float v) { return fminf((top - v) * scale, (float)(kBins - 1)); };  // (its whole part)
  bool binned = usable;
  unsigned long long total;
  __syncthreads();
  if (usable) {
    f.clear(sh.bins.amount, kBins);
    __syncthreads();
    f.template runs<2>([&](const float *x, int c, int) {
      constexpr int N = Piece<BF>::N;
      unsigned long long w[N];
#pragma unroll
      for (int e = 0; e < N; ++e) w[e] = quick(x[e]);
      if (last) {
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = place(x[e], c + e) >= last ? w[e] : 0;
      }
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (w[e]) atomicAdd(&sh.bins.amount[(int)bin(x[e])], w[e]);
    });
    __syncthreads();
    f.find(sh.bins.amount, kBins, ~0ull, total);
  } else {
    unsigned long long n = 0;
    f.template columns<true>([&](float v, int c) { n += place(v, c) >= last ? slow(v) : 0; });
    total = f.block_add(n);
  }
  // The place at which the sum from the first on reaches `target`, and the sum up to it.  `also` sees every column.
  auto where = [&](unsigned long long target, unsigned long long &upto, auto also) -> uint64_t {
    if (binned) {
      unsigned long long before;
      __syncthreads();
      const int b = f.find(sh.bins.amount, kBins, target, before);
      const float from = b, to = b + 1;
      auto wanted = [&](float v) {
        const float at = bin(v);
        return at >= from && at < to && v > -INFINITY;
      };
      f.begin();
      f.template runs<4>([&](const float *x, int c, int n) {
        bool any = false;
#pragma unroll
        for (int e = 0; e < Piece<BF>::N; ++e) {
          also(x[e], c + e);
          any |= wanted(x[e]);
        }
        if (any) f.mark(f.piece_of(c, n));
      });
      const int n = f.take([&](float v, int c) { return wanted(v) && place(v, c) >= last; });
      if (n <= kList) {
        f.sort(n, n);
        for (int i = tid; i < n; i += NT) sh.list[i] = quick(value_of(sh.sorted[i]));
        __syncthreads();
        if (wave == 0) {
          unsigned long long s;
          const int i = Sums(sh.list, n, lane).reach(target - before, s);
          if (lane == 0) { sh.found[0] = sh.sorted[i]; sh.found[1] = before + s; }
        }
        __syncthreads();
        upto = uniform_of(sh.found[1]);
        return uniform_of(sh.found[0]);
      }
    } else f.template columns<true>(also);
    binned = false;  // (reach takes the bins)
    const uint64_t at = f.template reach<true>(target, [&](float v, uint64_t q) -> unsigned long long { return q >= last ? mass(v) : 0; });
    unsigned long long s = 0;
    f.template columns<true>([&](float v, int c) {
      if (place(v, c) >= at) s += mass(v);
    });
    upto = f.block_add(s);
    return at;
  };
  if (p < 1.f) last = where(set.share(p, total), total, [](float, int) {});
  const uint64_t probable = m > 0.f ? place(least, (1 << kColumnBits) - 1) : 0;
  if (probable > last) {
    last = probable;
    unsigned long long s = 0;
    if (usable) f.columns([&](float v, int) { s += v >= least ? quick(v) : 0; });
    else f.template columns<true>([&](float v, int) { s += v >= least ? slow(v) : 0; });
    total = f.block_add(s);
  }
  unsigned long long upto;
  int n = 0;
  const float end = last ? value_of(last) : -3.402823466e38f;
  const int end_column = last ? column_of(last) : V;
  const uint64_t at = where(set.draw_at(total), upto, [&](float v, int c) { n += v > end || (v == end && c <= end_column); });
  n = (int)f.block_add((unsigned long long)n);
  if (tid == 0) {
    *token = column_of(at);
    if (logprob_out) *logprob_out = (float)slow.logarithm(value_of(at), total);
    if (kept) *kept = n;
  }
}

// A token of a row a workgroup.  Up to kTop candidates (top_k, or the largest alone) are listed and put in order, and one wave does the rest with them; other rows are weighed as
// a whole (above).  Few bytes and many steps, each waiting for the one before: the top 50 of 1 x 50257 fp32 in 8.9 us, of 4096 x 32000 bf16 in 72 (3.7 TB/s), top_p of 256 x
// 50257 fp32 in 50, 11 of them 64-bit exponentials and LDS additions.  With 16 pieces a thread 8 to 12 registers are spilled around the calls.
template <int BF, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void draw_kernel(const char *x, int64_t ld, int V, int bits, const float *uniform, twist_draw_rules rules, int32_t *tokens, float *logprobs, int32_t *kept) {
  Search<NT> &sh = shared<NT>();
  const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const device_bytes at_row = (device_bytes)(x + t * ld * Piece<BF>::ES);
  using R = Row<BF, NT, NV>;
  const int head = R::aligned((const char *)at_row, V);
  Settings set;
  set.u = uniform_of(uniform[t]);
  set.temp = rules.temperature ? uniform_of(rules.temperature[t]) : 1.f;
  set.p = rules.top_p ? uniform_of(rules.top_p[t]) : 1.f;
  set.m = rules.min_p ? uniform_of(rules.min_p[t]) : 0.f;
  set.k = rules.top_k ? uniform_of(rules.top_k[t]) : 0;
  const int k = min(V, set.temp > 0.f ? set.k : 1);
  if (k < 1 || k > kTop) {
    draw_of_many<BF, NT>(at_row, V, head, wave, bits, set, tokens + t, logprobs ? logprobs + t : nullptr, kept ? kept + t : nullptr);
    return;
  }
  R row(at_row, V, head, tid, wave);
  const Finder<BF, NT> f(sh, at_row, V, head, wave);
  f.prepare();
  float mine, top, low;
  extremes(row, sh, wave, lane, mine, top, low);
  const float from = bound_of(row, f, k, mine, top, low);
  int n = from > -INFINITY ? collect(row, f, from) : 0;
  if (n < k || n > kList) n = list_of_many<BF, NT>(at_row, V, head, wave, k);
  f.sort(n, k);
  const Weigher mass{top, 1.4426950408889634 / (double)set.temp, bits};
  for (int i = tid; i < k; i += NT) sh.list[i] = mass(value_of(sh.sorted[i]));
  __syncthreads();
  if (wave) return;
  const Sums sums(sh.list, k, lane);
  unsigned long long upto = sums.total, total;
  int count = 0;
  for (int i = lane; i < k; i += 64) count += value_of(sh.sorted[i]) > -INFINITY;
  count = wave_add(count);
  if (set.p < 1.f && count > 1) count = sums.reach(set.share(set.p, sums.total), upto) + 1;
  if (set.m > 0.f && count > 1) {
    const float least = mass.smallest(set.m, lane);
    int enough = 0;
    for (int i = lane; i < count; i += 64) enough += value_of(sh.sorted[i]) >= least;
    count = wave_add(enough);
    upto = sums.upto(count);
  }
  total = upto;
  const int i = sums.reach(set.draw_at(total), upto);
  if (lane == 0) {
    const uint64_t where = sh.sorted[i];
    tokens[t] = count ? column_of(where) : -1;
    if (logprobs) logprobs[t] = count ? (float)mass.logarithm(value_of(where), total) : -INFINITY;
    if (kept) kept[t] = count;
  }
}

// The list of `found` places put in order and its first n written (and k - n entries that are not there).
template <int BF, int NT>
__device__ __forceinline__ void write_top(Search<NT> &sh, int tid, int n, int k, int found, float hi, float lo, int32_t *ids, float *values) {
  const float scale = (kFew - 1) / (hi - lo);  // (of a list that reaches from or to infinity: 0, or no number)
  if (found > kByBins && scale > 0.f && scale < INFINITY) Finder<BF, NT>::sort_by_bins(sh, tid, found, hi, scale);
  else Finder<BF, NT>::sort(sh, tid, found, found);
  for (int i = tid; i < k; i += NT) {
    const uint64_t p = i < n ? sh.sorted[i] : 0;
    ids[i] = i < n ? column_of(p) : -1;
    values[i] = i < n ? value_of(p) : -INFINITY;
  }
}
// Over the workgroup: the sum, or the largest.  (Each kind once between two barriers of another step.)
template <int NT> __device__ __forceinline__ float block(Search<NT> &sh, int lane, int wave, float v, bool sum) {
  v = sum ? wave_add(v) : wave_max(v);
  float *all = sum ? sh.part : sh.most;
  if (lane == 0) all[wave] = v;
  __syncthreads();
  v = all[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v = sum ? v + all[w] : fmaxf(v, all[w]);
  return uniform_of(v);
}
// log2(e) over the temperature in 32 bits, with which differences of logits and their exponents are numbers of fp32, or else so large that their exponential is 0: not (no
// number) at temperatures next to nothing or to fp32's largest number.
__device__ __forceinline__ float exponent_of_2(double inv_temp) {
  const float c = (float)(1.4426950408889634 * inv_temp);
  return c > 1e-30f && c < 1e30f ? c : NAN;
}
// The log-sum-exp over the temperature of a row's columns behind the place `last`, -infinity where there are none.
template <int BF, int NT> __device__ __attribute__((noinline)) float rest_behind(device_bytes at_row, int V, int head, int wave, uint64_t last, double inv_temp) {
  Search<NT> &sh = shared<NT>();
  const Finder<BF, NT> f(sh, at_row, V, head, wave);
  auto others = [&](auto g) {
    f.columns([&](float v, int c) {
      if (v > -INFINITY && place(v, c) < last) g(v);
    });
  };
  float m = -INFINITY, s = 0.f;
  others([&](float v) { m = fmaxf(m, v); });
  m = block(sh, f.lane, wave, m, false);
  if (!(m > -INFINITY)) return m;
  const float c = exponent_of_2(inv_temp);
  if (c == c) others([&](float v) { s += v == m ? 1.f : __builtin_amdgcn_exp2f((v - m) * c); });
  else others([&](float v) { s += v == m ? 1.f : __builtin_amdgcn_exp2f((float)(((double)v - (double)m) * (1.4426950408889634 * inv_temp))); });
  s = block(sh, f.lane, wave, s, true);
  return (float)((double)m * inv_temp + log((double)s));
}

// The k largest of a row a workgroup: those above a bound that few columns reach, put in order; the pass that marks them also sums up the others, against the bound.  Bound by
// memory in the end, by the steps that wait for each other before that: the top 64 of 8192 x 50257 bf16 in 249 us (3.3 TB/s), the top 256 of 2048 x 32000 in 58.  With 16 pieces
// a thread 16 registers are spilled (8 with 256 threads and fp32) around the calls of the seldom ways, 32 or 64 bytes a thread that go to memory: 134 MB of the 139 that the
// first of these writes, 34 of 38 of the second.
template <int BF, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void top_kernel(const char *x, int64_t ld, int V, int k, double inv_temp, int32_t *ids, float *values, int64_t ldk, float *rest) {
  using R = Row<BF, NT, NV>;
  Search<NT> &sh = shared<NT>();
  const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = min(k, V);
  const device_bytes at_row = (device_bytes)(x + t * ld * Piece<BF>::ES);
  const int head = R::aligned((const char *)at_row, V);
  const float c = exponent_of_2(inv_temp);
  const Finder<BF, NT> f(sh, at_row, V, head, wave);
  float s = 0.f, from, largest;
  int found = 0;
  {
    R row(at_row, V, head, tid, wave);
    f.prepare();
    float mine, top, low;
    extremes(row, sh, wave, lane, mine, top, low);
    from = bound_of(row, f, n, mine, top, low);
    largest = top;
    // (without a bound nothing is marked, and what is summed up is no number)
    const float least = from > -INFINITY ? from : INFINITY;
    auto add = [&](float v) { s += __builtin_amdgcn_exp2f(fmaxf((v - least) * c, -126.f)); };  // (also of no number)
    row.each([&](const Piece<BF> &y, int v) {
      Piece<BF> z = y;
      if (y.most() >= least) {
        f.mark(v);
        uint32_t above = 0;
#pragma unroll
        for (int e = 0; e < Piece<BF>::N; ++e) above |= (uint32_t)(y[e] >= least) << e;
        z.clear(above);
      }
#pragma unroll
      for (int e = 0; e < Piece<BF>::N; ++e) add(z[e]);
    });
    if (row.xl >= least) f.mark(row.pieces + tid);
    else add(row.xl);
    found = f.take([&](float v, int) { return v >= least; });
  }
  const bool quick = from > -INFINITY && found >= n && found <= kList;
  if (!quick) found = list_of_many<BF, NT>(at_row, V, head, wave, n);
  write_top<BF, NT>(sh, tid, n, k, found, quick ? largest : sh.hi, quick ? from : sh.lo, ids + t * ldk, values + t * ldk);
  if (!rest) return;
  // the list's others may lie far above the bound: then against the largest of them
  const float ref = uniform_of(found > n ? value_of(sh.sorted[n]) : from);
  s *= __builtin_amdgcn_exp2f((from - ref) * c);
  for (int i = n + tid; i < found; i += NT) s += __builtin_amdgcn_exp2f((value_of(sh.sorted[i]) - ref) * c);
  s = block(sh, lane, wave, s, true);
  float r = (float)((double)ref * inv_temp + log((double)s));
  if (!quick || !(s > 0.02f)) r = rest_behind<BF, NT>(at_row, V, head, wave, uniform_of(sh.sorted[n - 1]), inv_temp);  // (the others are far below the bound, there is none, or c is no number)
  if (tid == 0) rest[t] = r;
}

// The kernel whose registers hold a row.  A CU holds one workgroup of 1024 threads, two of 512 or four of 256: while every CU has a row at most, 1024 threads are through it
// sooner, with more rows it is several rows side by side that keep the memory busy while each has its steps to wait for (drawing from the top 50, bf16: 256 x 32000 10.6 us with
// 1024 threads, 13.3 with 256; 512 x 32000 20.4 and 17.3, 4096 x 32000 147 and 77; 4096 x 50257 172 and, with 512, 120; fp32 4096 x 16384 127 and 72, 4096 x 32000 182 and 128).
// The largest 64 of a row likewise.
constexpr int kManyRows = 256;  // one for every CU
#define ROWS_BF16(LAUNCH)                              \
  do {                                                 \
    if (V <= 4 * 8 * 256) LAUNCH(1, 256, 4);           \
    else if (T > kManyRows && V <= 16 * 8 * 256) LAUNCH(1, 256, 16); \
    else if (T > kManyRows && V <= 16 * 8 * 512) LAUNCH(1, 512, 16); \
    else if (V <= 4 * 8 * 1024) LAUNCH(1, 1024, 4);    \
    else if (V <= 8 * 8 * 1024) LAUNCH(1, 1024, 8);    \
    else LAUNCH(1, 1024, 0);                           \
  } while (0)
#define ROWS_F32(LAUNCH)                               \
  do {                                                 \
    if (V <= 4 * 4 * 256) LAUNCH(0, 256, 4);           \
    else if (T > kManyRows && V <= 16 * 4 * 256) LAUNCH(0, 256, 16); \
    else if (T > kManyRows && V <= 16 * 4 * 512) LAUNCH(0, 512, 16); \
    else if (V <= 4 * 4 * 1024) LAUNCH(0, 1024, 4);    \
    else if (V <= 16 * 4 * 1024) LAUNCH(0, 1024, 16);  \
    else LAUNCH(0, 1024, 0);                           \
  } while (0)

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
#define DRAW(BF, NT, NV) \
  hipLaunchKernelGGL((draw_kernel<BF, NT, NV>), dim3(T), dim3(NT), 0, ctx->stream, static_cast<const char *>(logits), ld, V, bits, uniform, r, tokens, logprobs, kept)
  if (ctx->d.dtype == TWIST_BF16 && !logits_f32) ROWS_BF16(DRAW);
  else ROWS_F32(DRAW);
#undef DRAW
  TW_HIP(ctx, hipGetLastError());
  return TWIST_OK;
}

twist_status twist_check_top(twist_ctx *ctx, const char *who, int64_t ld, int T, int k, float temperature, int64_t ldk) {
  TW_TRY(check_rows(ctx, who, ld, T));
  if (k < 1 || k > kTop) TW_FAIL(ctx, TWIST_ESHAPE, "%s: lists of %d entries (1 to %d)", who, k, kTop);
  if (ldk < k) TW_FAIL(ctx, TWIST_ESHAPE, "%s: rows of the lists overlap", who);
  if (!(temperature > 0.f && temperature < INFINITY)) TW_FAIL(ctx, TWIST_EINVAL, "%s: the temperature must be above 0 and finite", who);
  return TWIST_OK;
}

extern "C" twist_status twist_top_logits_raw(twist_ctx *ctx, const void *logits, int64_t ld, int32_t logits_f32, int32_t T, int32_t k, float temperature, int32_t *ids,
                                             float *values, int64_t ldk, float *rest) {
  const char *who = "twist_top_logits_raw";
  if (!ctx || !logits || !ids || !values) TW_FAIL(ctx, TWIST_EINVAL, "%s: null argument", who);
  TW_TRY(twist_check_top(ctx, who, ld, T, k, temperature, ldk));
  const int V = ctx->d.vocab;
  const double inv = 1.0 / (double)temperature;
#define TOP(BF, NT, NV) \
  hipLaunchKernelGGL((top_kernel<BF, NT, NV>), dim3(T), dim3(NT), 0, ctx->stream, static_cast<const char *>(logits), ld, V, k, inv, ids, values, ldk, rest)
  if (ctx->d.dtype == TWIST_BF16 && !logits_f32) ROWS_BF16(TOP);
  else ROWS_F32(TOP);
#undef TOP
  TW_HIP(ctx, hipGetLastError());
  return TWIST_OK;
}
