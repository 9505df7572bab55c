// The rotation of one row's heads by a wave, shared by the standalone rotary
// kernel and the cache append.
#pragma once
#include "kv8_device.h"

// Whether a view's heads can be taken 16 bytes at a time: base, strides and the
// table's pairs keep every piece aligned and whole.
inline bool rope_vectors(int dtype, const HeadView& x, int hd, const RopeTable& t) {
  const int e = dtype == 1 ? 8 : 4;   // elements of 16 bytes
  const int piece = t.layout ? 2 * t.pairs : t.pairs;   // rotated elements side by side
  return (uintptr_t)x.p % 16 == 0 && x.row % e == 0 && x.head % e == 0 && hd % e == 0 && piece % e == 0 &&
         (hd - 2 * t.pairs) % e == 0 && (uintptr_t)t.cos % 16 == 0 && (uintptr_t)t.sin % 16 == 0 &&
         (t.layout == 0 || t.pairs % 4 == 0);
}

// Unit u of a head: N elements of the lower and of the upper half (half
// layout), N / 2 pairs (interleaved), or N copied elements past the pairs.
template <typename T, int VEC, int LAYOUT>
struct RopeUnit {
  static constexpr int N = LAYOUT == 1 && VEC == 1 ? 2 : VEC;
  static constexpr bool V = VEC > 1;
  float c[N], s[N];   // interleaved: N / 2 of them
  int at, n;          // element offset; 0 turned, 1 copied, 2 none
  int m;

  __device__ __forceinline__ void start(const RopeTable& t, int pos, float sign, int u, int hd) {
    m = t.pairs;
    const int ru = (LAYOUT ? 2 * m : m) / N;
    n = u < ru ? 0 : 1;
    at = u < ru ? u * N : 2 * m + (u - ru) * N;
    if (n) return;
    constexpr int C = LAYOUT ? N / 2 : N;
    const int i0 = LAYOUT ? at / 2 : at;
    float cc[C], ss[C];
    if ((unsigned)pos < (unsigned)t.n_pos) {
      ld_elems<C, V>(t.cos + (int64_t)pos * m + i0, cc);
      ld_elems<C, V>(t.sin + (int64_t)pos * m + i0, ss);
    } else {                      // no such position: the values are NaN
#pragma unroll
      for (int i = 0; i < C; ++i) cc[i] = ss[i] = __uint_as_float(0x7FC00000u);
    }
#pragma unroll
    for (int i = 0; i < C; ++i) { c[i] = cc[i]; s[i] = ss[i] * sign; }
  }
  __device__ __forceinline__ void load(const T* x, float (&a)[N], float (&b)[N]) const {
    ld_elems<N, V>(x + at, a);
    if (LAYOUT == 0 && n == 0) ld_elems<N, V>(x + m + at, b);
  }
  __device__ __forceinline__ void store(T* y, float (&a)[N], float (&b)[N]) const {
    if (n == 0) {
      if constexpr (LAYOUT == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float p = turn_lo(a[i], b[i], c[i], s[i]), q = turn_hi(a[i], b[i], c[i], s[i]);
          a[i] = p;
          b[i] = q;
        }
        st_elems<N, V>(y + m + at, b);
      } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          const float p = turn_lo(a[i], a[i + 1], c[i / 2], s[i / 2]), q = turn_hi(a[i], a[i + 1], c[i / 2], s[i / 2]);
          a[i] = p;
          a[i + 1] = q;
        }
      }
    }
    st_elems<N, V>(y + at, a);
  }
};

// Turns (sign -1: back) the heads of one row.  One wave; y may be x.
template <typename T, int VEC, int LAYOUT>
__device__ __forceinline__ void rope_row(const T* x, int64_t x_head, T* y, int64_t y_head, int heads, int hd,
                                         const RopeTable& t, int pos, float sign, int lane) {
  using Unit = RopeUnit<T, VEC, LAYOUT>;
  constexpr int N = Unit::N, INFLIGHT = 4;
  const int units = (LAYOUT ? 2 * t.pairs : t.pairs) / N + (hd - 2 * t.pairs) / N;
  Unit un;
  if (units <= 64) {   // a lane keeps its unit and goes from head to head
    const int per = 64 / units, h0 = lane / units;
    if (h0 >= per) return;
    un.start(t, pos, sign, lane % units, hd);
    for (int h = h0; h < heads; h += per * INFLIGHT) {
      float a[INFLIGHT][N], b[INFLIGHT][N];
#pragma unroll
      for (int i = 0; i < INFLIGHT; ++i)
        if (h + i * per < heads) un.load(x + (h + i * per) * x_head, a[i], b[i]);
#pragma unroll
      for (int i = 0; i < INFLIGHT; ++i)
        if (h + i * per < heads) un.store(y + (h + i * per) * y_head, a[i], b[i]);
    }
  } else {
    for (int u = lane; u < units; u += 64) {
      un.start(t, pos, sign, u, hd);
      for (int h = 0; h < heads; ++h) {
        float a[N], b[N];
        un.load(x + h * x_head, a, b);
        un.store(y + h * y_head, a, b);
      }
    }
  }
}
