// A row of logits in a workgroup's registers, for the kernels that go through it more than once.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));
// Memory of the device, said to be: what a function that is not inlined is given could be LDS as well, and its loads would be waited for with those
typedef const __attribute__((address_space(1))) char *device_bytes;

// Sixteen bytes of a row, as floats: eight of bf16, four of fp32.
template <int BF> struct Piece {
  static constexpr int N = BF ? 8 : 4, ES = BF ? 2 : 4;
  u32x4v u;
  __device__ __forceinline__ void load(device_bytes p) { u = *(const __attribute__((address_space(1))) u32x4u *)p; }  // (from any element on)
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
  __device__ __forceinline__ float most() const {
    float m = fmaxf((*this)[0], (*this)[1]);
#pragma unroll
    for (int e = 2; e < N; ++e) m = fmaxf(m, (*this)[e]);
    return m;
  }
};
template <int BF> __device__ __forceinline__ float load1(device_bytes row, int c) {
  if (BF) return __uint_as_float((uint32_t)((const __attribute__((address_space(1))) uint16_t *)row)[c] << 16);
  return ((const __attribute__((address_space(1))) float *)row)[c];
}
template <int BF> __device__ __forceinline__ void store1(char *row, int64_t c, float v) {
  if (BF) reinterpret_cast<__bf16 *>(row)[c] = (__bf16)v;  // round to nearest even
  else reinterpret_cast<float *>(row)[c] = v;
}

// v of another lane, by the data-parallel moves of the vector unit (an eighth of what a trip through LDS takes): CTRL row_shr:1 to 8 (0x111 ..), row_bcast:15 and :31 (0x142,
// 0x143) for the rows of ROWS; lanes that have no such neighbour get `none`.
template <int CTRL, int ROWS, class T> __device__ __forceinline__ T moved(T none, T v) {
  constexpr int W = sizeof(T) / 4;
  uint32_t a[W], b[W];
  __builtin_memcpy(a, &none, sizeof(T));
  __builtin_memcpy(b, &v, sizeof(T));
#pragma unroll
  for (int w = 0; w < W; ++w) a[w] = __builtin_amdgcn_update_dpp(a[w], b[w], CTRL, ROWS, 0xf, false);
  __builtin_memcpy(&v, a, sizeof(T));
  return v;
}
// v of lane 63, in all lanes
template <class T> __device__ __forceinline__ T last_of(T v) {
  constexpr int W = sizeof(T) / 4;
  uint32_t a[W];
  __builtin_memcpy(a, &v, sizeof(T));
#pragma unroll
  for (int w = 0; w < W; ++w) a[w] = __builtin_amdgcn_readlane(a[w], 63);
  __builtin_memcpy(&v, a, sizeof(T));
  return v;
}
// Sums over the lanes up to each: along the rows of 16, then over them
template <class T> __device__ __forceinline__ T wave_sums(T v) {
  const T zero = 0;
  v += moved<0x111, 0xf>(zero, v);
  v += moved<0x112, 0xf>(zero, v);
  v += moved<0x114, 0xf>(zero, v);
  v += moved<0x118, 0xf>(zero, v);
  v += moved<0x142, 0xa>(zero, v);
  v += moved<0x143, 0xc>(zero, v);
  return v;
}
template <class T> __device__ __forceinline__ T wave_add(T v) { return last_of(wave_sums(v)); }
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, moved<0x111, 0xf>(v, v));
  v = fmaxf(v, moved<0x112, 0xf>(v, v));
  v = fmaxf(v, moved<0x114, 0xf>(v, v));
  v = fmaxf(v, moved<0x118, 0xf>(v, v));
  v = fmaxf(v, moved<0x142, 0xa>(v, v));
  v = fmaxf(v, moved<0x143, 0xc>(v, v));
  return last_of(v);
}

// The row as NV pieces a thread, beginning where an address is aligned (`head` columns on); the columns before and behind the pieces, `ends` of them, are a thread's each (xl,
// column `end`).  Pieces beyond the row hold -infinity.  NV = 0: rows that NT threads cannot hold are read again for every pass.
template <int BF, int NT, int NV> struct Row {
  using P16 = Piece<BF>;
  static constexpr int N = P16::N, ES = P16::ES, NW = NT / 64;
  P16 x[NV ? NV : 1];
  float xl;
  device_bytes first;
  int head, pieces, mine, ends, end, tid;
  __device__ __forceinline__ Row(device_bytes row, int V, int head_, int tid_, int wave) { fetch(row, V, head_, tid_, wave); }
  __device__ __forceinline__ void fetch(device_bytes row, int V, int head_, int tid_, int wave) {
    tid = tid_;
    head = head_;
    pieces = (V - head) / N;
    mine = pieces - 64 * wave;  // u NT >= mine: the wave's piece u lies beyond the row
    ends = V - pieces * N;
    end = tid < head ? tid : pieces * N + tid;
    first = row + head * ES;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      x[u].u = P16::none();
      if (u * NT + tid < pieces) x[u].load(first + (int64_t)(u * NT + tid) * 16);
    }
    xl = tid < ends ? load1<BF>(row, end) : -INFINITY;
  }
  __device__ __forceinline__ static int aligned(const void *row, int V) { return min(V, (int)(-(reinterpret_cast<uintptr_t>(row) / ES) & (N - 1))); }
  // f(piece, its number) for all of the thread's pieces
  template <class F> __device__ __forceinline__ void each(F f) {
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
        f(y, v);
      }
    }
  }
};

}  // namespace
