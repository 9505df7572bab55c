// Sampling from given logits and given uniform numbers: temperature, top-k, top-p,
// min-p.
//
// Weights are w = exp((z - max z) / T).  Tokens in order of z, ties by id: top-k keeps
// the first k, top-p those before which less than p of the k's weight lies, min-p
// those with z >= max z + T ln(min_p).  Each keeps a beginning of that order, so all
// together keep one: the tokens up to a border (z, id).  The draw is the first token,
// by id, at which the kept weights' running sum passes u times their sum.
//
// A vocabulary has as many places where a draw turns on the running sum, so that sums
// which are 1e-8 off, as those of fp32 weights are, draw another token in one row of a
// thousand.  Weights are therefore fp64, by a polynomial of their own (Exp2, 1e-12):
// 14 instructions a token, which still fit under the bytes of fp32 logits.  Where
// something is cut the weights are whole numbers, w 2^42 to nearest: their sums do not
// depend on any order, so atomics give the same draw on every run.
//
// Launches:
// * scan, a wave pairs of segments of 512 tokens: maximum, and sum of weights with respect
//   to it; maxima of strips of 64.  It streams the logits once.
// * where nothing can be cut: plain, a workgroup a row.  The segment at which the running
//   sum passes, then the token.
// * only where top-p or min-p may cut rows without top-k that one workgroup would be slow
//   at: bins and collect (some workgroups a row, each a part of it).  The bins find the row's sum and the least z that can be
//   kept, and add up weights by z; collect finds the bin in which the border of top-p lies,
//   sums what each part keeps above it, and lists the tokens in it.
// * pick, a workgroup a row: the border, then where the running sum passes.
// All after the scan look only at strips that can hold kept tokens:
// * weights below 2^-43 of the largest count nothing;
// * k segments, or strips, with a maximum of t or more hold k tokens of t or more, so the
//   border of top-k lies there or above;
// * what lies below t weighs no more than the segments whose maximum is below t and
//   512 w(t) of each other, and where that is at most 1 - p of all, the border of
//   top-p lies at t or above.
#include <algorithm>
#include <type_traits>

#include "kv8_device.h"

namespace {

typedef unsigned long long u64;

constexpr int SEG = 512;              // tokens of a segment
constexpr int MAX_SEGS = 2048;        // of a row: 2^20 tokens
constexpr int STRIP = 64;             // tokens of a strip
constexpr int STRIPS = SEG / STRIP;
constexpr int STEPS = 512;            // that the octaves are told apart in for top-k
constexpr int SCAN_WAVES = 4;
constexpr int SCAN_FILL = 32768;      // waves of the scan, where there are segments for so many
constexpr int PART = 256;             // threads of a part of a row's histogram
// threads of a row's pick: 8, 64 and 505 rows take 12, 19, 16 us; by 256 threads 16, 23, 18; by 1024 12, 21, 27
constexpr int PICK = 512;
constexpr int BINS = 1024;            // of z in a row's histogram
constexpr int LIST = 4096;            // tokens that a row's list holds
constexpr int OWN_BINS = 1024;        // tokens past which the pick goes by a histogram of its own (4000: 18-20 us, by a list 25-27)
constexpr int ROWS_FULL = 256;        // rows that keep the chip busy, a workgroup each
constexpr int ID_BITS = 20;
constexpr double LOG2E = 1.4426950408889634;
constexpr double FIXED_ONE = 4398046511104.0;   // 2^42
constexpr float FIXED_OCTAVES = 43.5f;          // weights below 2^-43 are 0 in whole numbers

// Octaves of weight per logit; temperature 0 reports at 1.
__device__ __forceinline__ double octaves_per_logit(const DrawArgs& A, int r) {
  if (!A.temperature_rows) return A.c;
  const float t = A.temperature_rows[r];
  return t == 0.f ? LOG2E : LOG2E / (double)t;
}

// Settings of a row.
struct RowOpts {
  double temperature, top_p, min_p;
  int top_k;
  bool by_k, by_p, by_min;
  double c;
};
__device__ __forceinline__ RowOpts row_opts(const DrawArgs& A, int r) {
  RowOpts o;
  o.temperature = A.temperature_rows ? (double)A.temperature_rows[r] : A.temperature;
  o.top_k = A.top_k_rows ? A.top_k_rows[r] : A.top_k;
  o.top_p = A.top_p_rows ? (double)A.top_p_rows[r] : A.top_p;
  o.min_p = A.min_p_rows ? (double)A.min_p_rows[r] : A.min_p;
  o.by_k = o.top_k > 0 && o.top_k < A.vocab;
  o.by_p = o.top_p < 1.0;
  o.by_min = o.min_p > 0.0;
  o.c = octaves_per_logit(A, r);
  return o;
}
__device__ __forceinline__ bool usable(const RowOpts& o) {
  return o.temperature >= 0.0 && o.temperature < (double)INFINITY && o.top_p == o.top_p && o.min_p == o.min_p;
}

// 2^t for t in [-1000, 1000]: 2^n times a polynomial of degree 8 that interpolates 2^f
// at the Chebyshev points of [-1/2, 1/2], 1.1e-12 relative.  Its coefficients are held in
// scalar registers: as literals they were moved into vector ones again for every segment.
struct Exp2 {
  static constexpr int N = 8;
  u64 a[N];
  __device__ __forceinline__ Exp2() {
    constexpr double coefficients[N] = {1.3255224884799127e-06, 1.5310079402383103e-05, 0.00015403455852419016,
                                        0.0013333450568000008,  0.00961812915940262,    0.05550410941205934,
                                        0.2402265069581299,     0.6931471805459335};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      a[i] = __builtin_bit_cast(u64, coefficients[i]);
      asm("" : "+s"(a[i]));
    }
  }
  static constexpr double SHIFTER = 6755399441055744.0;       // 1.5 * 2^52: the low bits of a sum with it are
                                                               // the other part, to nearest
  // 2^f times 2 to the whole number in the low bits of s
  __device__ __forceinline__ double at(double f, double s) const {
    double p = __builtin_bit_cast(double, a[0]);
#pragma unroll
    for (int i = 1; i < N; ++i) p = fma(p, f, __builtin_bit_cast(double, a[i]));
    p = fma(p, f, 1.0);
    u32x2_t w = __builtin_bit_cast(u32x2_t, p);               // into the exponent: of the high word alone
    w[1] += __builtin_bit_cast(u32x2_t, s)[0] << 20;
    return __builtin_bit_cast(double, w);
  }
  __device__ __forceinline__ double operator()(double t) const {
    const double s = t + SHIFTER;
    return at(t - (s - SHIFTER), s);
  }
};
// The weight of z with respect to top (finite, no less): octaves below 1000 count nothing.
__device__ __forceinline__ double weight_of(const Exp2& exp2, float z, float top, double c) {
  return exp2(fmax(((double)z - (double)top) * c, -1000.0));
}
// w 2^42 to nearest.
__device__ __forceinline__ u64 fixed_of(double w) {
  return __builtin_bit_cast(u64, fma(w, FIXED_ONE, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;   // 2^52 + w 2^42
}

// NaN where either is.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// A value of another lane, 0 where there is none or the lane's row of 16 is not in ROWS.
template <int CTRL, int ROWS, typename V>
__device__ __forceinline__ V shifted(V v) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, true));
  } else {
    const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
    return __builtin_bit_cast(V, u32x2_t{(uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[0], CTRL, ROWS, 0xF, true),
                                         (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[1], CTRL, ROWS, 0xF, true)});
  }
}
// Maxima over lanes go by whole numbers in the order of z, NaN above all: one lane move
// and comparison a step.
__device__ __forceinline__ int rank_of(float z) {
  const int u = __float_as_int(z);
  return z == z ? u ^ (u >> 31 & 0x7FFFFFFF) : INT32_MAX;
}
__device__ __forceinline__ float of_rank(int k) {
  return k == INT32_MAX ? __uint_as_float(0x7FC00000u) : __int_as_float(k ^ (k >> 31 & 0x7FFFFFFF));
}
template <int CTRL>
__device__ __forceinline__ int max_moved(int v) {
  return max(v, __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false));
}
// Eight tokens of a row from the i-th on; -inf past its end.
template <typename T, bool VEC>
struct Eight {
  typedef T vec __attribute__((ext_vector_type(8), aligned(16)));
  vec t;
  __device__ __forceinline__ void load_whole(const T* p) { t = *reinterpret_cast<const vec*>(p); }
  __device__ __forceinline__ void load(const T* p, int i, int n) {
    if constexpr (sizeof(T) == 2) t = (vec)(T)0xFF80;
    else t = (vec)-INFINITY;
    if (i >= n) return;
    if (VEC && i + 8 <= n) {
      t = *reinterpret_cast<const vec*>(p + i);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i + e < n) t[e] = p[i + e];
    }
  }
  __device__ __forceinline__ float operator[](int e) const {
    const T x = t[e];
    return ld_f32<T>(&x);
  }
  // a bit for each that is t0 or more; tokens past the vocabulary are -inf
  __device__ __forceinline__ uint32_t from(float t0) const {
    uint32_t hits = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) hits |= (uint32_t)((*this)[e] >= t0 && (*this)[e] > -INFINITY) << e;
    return hits;
  }
  __device__ __forceinline__ float at(int k) const {
    float x = (*this)[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) x = e == k ? (*this)[e] : x;
    return x;
  }
};

// Where 2^(z c) of a segment's tokens is not out of all bounds, their weights are taken with
// respect to the whole octave next to the maximum's m c, else to m itself.
__device__ __forceinline__ bool by_octave(float m, double c) {
  return fabs((double)m * c) < 1024.0 && c > 1e-30 && c < 1e30 && fabsf(m) < 1e38f;
}
// A segment's weight with respect to the row's maximum.
__device__ __forceinline__ double share_of(const Exp2& exp2, float m, double s, float zmax, double c) {
  if (m == -INFINITY) return 0.0;
  const double t = by_octave(m, c) ? fma(-(double)zmax, c, rint((double)m * c)) : ((double)m - (double)zmax) * c;
  return s * exp2(fmax(t, -1000.0));
}

// ---------------------------------------------------------------- scan
// A wave goes through `per` pairs of segments, whose loads are on their way together; the
// halves of the wave then take the pair's lane moves.  The code is kept small here and below:
// each kernel starts with none of it in the instruction cache, and lines that are run once
// cost more than what is in them (the pick of 505 rows 35 us with 94 KB of code, 22 with 39).
// 512 rows of 151936 fp32 logits 60 us, 5.2 TB/s: fp64 instructions, 14 a token, take as long
// as the read; 64 rows of 152064 bf16 ones 12 us, those alone.
// The next pair held in registers ahead 64 us, segments one by one 70.
template <typename T, bool VEC, bool CUT>
__global__ __launch_bounds__(64 * SCAN_WAVES) void k_draw_scan(DrawArgs A, int segs, unsigned per_row, unsigned items,
                                                                 unsigned per) {
  const int lane = threadIdx.x & 63;
  unsigned item = (blockIdx.x * SCAN_WAVES + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6))) * per;
  if (item >= items) return;
  const unsigned end = min(items, item + per);
  unsigned r = item / per_row;
  int s = (int)(item - r * per_row) * 2;
  const T* z = (const T*)A.logits + r * A.row;
  const Exp2 exp2;
  double c = octaves_per_logit(A, r);
#pragma unroll 1
  for (;;) {
    Eight<T, VEC> v[2];
    const int64_t at = (int64_t)r * segs + s;
    if (VEC && (s + 2) * SEG <= A.vocab) {
      v[0].load_whole(z + s * SEG + 8 * lane);
      v[1].load_whole(z + (s + 1) * SEG + 8 * lane);
    } else {
      v[0].load(z, s * SEG + 8 * lane, A.vocab);
      v[1].load(z, (s + 1) * SEG + 8 * lane, A.vocab);
    }
    int rank[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float top = v[j][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = max_nan(top, v[j][e]);
      rank[j] = rank_of(top);
    }
    auto step = [&](auto ctrl) {
      rank[0] = max_moved<decltype(ctrl)::value>(rank[0]);
      rank[1] = max_moved<decltype(ctrl)::value>(rank[1]);
    };
    if constexpr (CUT) {                          // of eight lanes, in lanes 7, 15, ..
      step(std::integral_constant<int, 0x111>{});
      step(std::integral_constant<int, 0x112>{});
      step(std::integral_constant<int, 0x114>{});
      if ((lane & 7) == 7) {
        float* strip = A.strip_m + at * STRIPS + (lane >> 3);
        strip[0] = of_rank(rank[0]);
        if (s + 1 < segs) strip[STRIPS] = of_rank(rank[1]);
      }
    }
    // the halves of the wave take a segment each
    auto swapped = __builtin_amdgcn_permlane32_swap((uint32_t)rank[0], (uint32_t)rank[1], false, false);
    int both = max((int)swapped[0], (int)swapped[1]);
    if constexpr (!CUT) {
      both = max_moved<0x111>(both);
      both = max_moved<0x112>(both);
      both = max_moved<0x114>(both);
    }
    both = max_moved<0x118>(both);
    both = max_moved<0x142>(both);
    float m[2] = {of_rank(__builtin_amdgcn_readlane(both, 31)), of_rank(__builtin_amdgcn_readlane(both, 63))};
    if (s + 1 >= segs) m[1] = m[0];
    double sum[2] = {0.0, 0.0};
    if (by_octave(m[0], c) && by_octave(m[1], c)) {
      // z c, and the whole octave next to it in the low bits of s; where z is 1000 octaves
      // down already it goes no further
      const float reach = 1000.f * __builtin_amdgcn_rcpf((float)c);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float least = m[j] - reach;
        const double shifter = Exp2::SHIFTER - rint((double)m[j] * c);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double x = (double)__builtin_amdgcn_fmed3f(v[j][e], least, 3.0e38f), n = fma(x, c, shifter);
          sum[j] += exp2.at(fma(x, c, shifter - n), n);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (m[j] > -INFINITY && m[j] < INFINITY) {   // else the sum is not looked at, or nothing
          const bool octave = by_octave(m[j], c);
          const double top = rint((double)m[j] * c);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const double z = (double)v[j][e], t = octave ? fma(z, c, -top) : (z - (double)m[j]) * c;
            sum[j] += exp2(fmax(t, -1000.0));
          }
        }
    }
    const u32x2_t a = __builtin_bit_cast(u32x2_t, sum[0]), b = __builtin_bit_cast(u32x2_t, sum[1]);
    const auto low = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false);
    const auto high = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
    double all = __builtin_bit_cast(double, u32x2_t{low[0], high[0]}) + __builtin_bit_cast(double, u32x2_t{low[1], high[1]});
    all += shifted<0x111, 0xF>(all);
    all += shifted<0x112, 0xF>(all);
    all += shifted<0x114, 0xF>(all);
    all += shifted<0x118, 0xF>(all);
    all += shifted<0x142, 0xF>(all);
    const int half = lane >> 5;
    if ((lane & 31) == 31 && s + half < segs) {
      A.seg_m[at + half] = half ? m[1] : m[0];
      A.seg_s[at + half] = all;
    }
    if (CUT && A.bins) {                          // the histogram begins empty
      const int share = (BINS + (int)per_row - 1) / (int)per_row, b0 = s / 2 * share;
      u64* bins = A.bins + (at - s) / segs * BINS;
#pragma unroll 1
      for (int i = b0 + lane; i < min(b0 + share, BINS); i += 64) bins[i] = 0;
    }
    if (++item == end) return;
    s += 2;
    if (s >= segs) {
      s = 0;
      ++r;
      z += A.row;
      c = octaves_per_logit(A, r);
    }
  }
}

// ---------------------------------------------------------------- a row
// Order of z as whole numbers, and back.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z == 0.f ? 0.f : z);       // -0 is 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
// A token's place in the order, its own: a larger one comes first.  bf16's are 36 bits
// wide, so that few distinct values with many ids each do not leave most windows empty.
template <typename T>
struct Places {
  static constexpr int DROP = sizeof(T) == 2 ? 16 : 0;
  static __device__ __forceinline__ u64 of(float z, int id) {
    return (u64)(key_of(z) >> DROP) << ID_BITS | (uint32_t)((1 << ID_BITS) - 1 - id);
  }
  static __device__ __forceinline__ float z(u64 place) {
    const uint32_t k = (uint32_t)(place >> ID_BITS) << DROP;
    return of_key(DROP && !(k & 0x80000000u) ? k | 0xFFFFu : k);
  }
  static __device__ __forceinline__ int id(u64 place) { return (1 << ID_BITS) - 1 - (int)(place & ((1 << ID_BITS) - 1)); }
  // the lowest of a z that is not below t
  static __device__ __forceinline__ u64 from(float t) {
    const u64 p = (u64)(key_of(t) >> DROP) << ID_BITS;
    return z(p) < t ? p + (1ull << ID_BITS) : p;
  }
};

template <typename V>
__device__ __forceinline__ V wave_prefix(V v) {                      // inclusive
  v += shifted<0x111, 0xF>(v);
  v += shifted<0x112, 0xF>(v);
  v += shifted<0x114, 0xF>(v);
  v += shifted<0x118, 0xF>(v);
  v += shifted<0x142, 0xA>(v);
  v += shifted<0x143, 0xC>(v);
  return v;
}
// Over a workgroup of N threads; `red` holds a value a wave.
template <int N, typename V>
__device__ __forceinline__ V group_prefix(V v, V* red, V* total) {   // inclusive
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  v = wave_prefix(v);
  __syncthreads();
  if (lane == 63) red[w] = v;
  __syncthreads();
  V all = 0;
#pragma unroll
  for (int i = 0; i < N / 64; ++i) {
    if (i < w) v += red[i];
    all += red[i];
  }
  *total = all;
  return v;
}
template <int N>
__device__ __forceinline__ int group_min(int v, int* red) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  v = -v;
  v = max_moved<0x111>(v);
  v = max_moved<0x112>(v);
  v = max_moved<0x114>(v);
  v = max_moved<0x118>(v);
  v = max_moved<0x142>(v);
  v = max_moved<0x143>(v);
  __syncthreads();
  if (lane == 63) red[w] = -v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < N / 64; ++i) v = min(v, red[i]);
  return v;
}
template <typename V>
__device__ __forceinline__ V lane_of(V v, int lane) {
  const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
  return __builtin_bit_cast(V, u32x2_t{(uint32_t)__builtin_amdgcn_readlane((int)w[0], lane),
                                       (uint32_t)__builtin_amdgcn_readlane((int)w[1], lane)});
}
__device__ __forceinline__ int first_lane(uint64_t mask) { return __ffsll((unsigned long long)mask) - 1; }
__device__ __forceinline__ int last_lane(uint64_t mask) { return 63 - __clzll((long long)mask); }

// Bin of z: falls as z grows.  The bins share out what lies between t0 and the maximum, and
// hold a sixteenth of an octave of weight at most.
__device__ __forceinline__ float bins_per_logit(float zmax, float t0, float c) {
  return fminf(fmaxf(16.f * c, (float)(BINS - 1) / (zmax - t0)), 3.0e38f);
}
__device__ __forceinline__ int bin_of(float z, float zmax, float per) { return (int)fminf((zmax - z) * per, (float)(BINS - 1)); }
__device__ __forceinline__ float bin_factor(double c) { return (float)fmin(c, 3.0e38); }
// Weight, or u of it, at which top-p ends: the first token is always kept.
__device__ __forceinline__ double mass_limit(const RowOpts& o, double all) { return fmax((double)o.top_p * all, 0.5); }
// Whether the pick deals with every row alone.  Top-p by several workgroups a row takes
// three launches, by one a histogram of its own: 2 to 150 rows of 5000 28-32 and 22-23 us, of
// 16000 28-36 and 28-31, of 32000 29-46 and 40-46.  Where rows are enough for all units and
// have k of their own, which may leave the launches few of them, it pays further: 505 rows of
// 20000 bf16 tokens, all by top-p alone, half, a tenth of them, 57, 50, 42 us and 42, 40, 35;
// of 32000 65, 57, 48 and 57, 56, 50 (near-uniform logits 78, 69, 54 and 72, 71, 70); but of
// 50257 138, 117, 93 and 158, 145, 133, of 65536 100, 82, 70 and 111, 106, 86.
__host__ __device__ __forceinline__ bool alone(const DrawArgs& A) {
  return A.vocab <= (A.rows >= ROWS_FULL && A.top_k_rows ? 1 << 15 : 1 << 14);
}
// Which rows several workgroups look at, by a histogram.  top-k's tokens are few.  min-p's
// border is known, but summing up what it leaves takes one workgroup a row long where that
// is most of it (64 rows of 152064: 77 us, by several 43).
__device__ __forceinline__ bool by_bins(const RowOpts& o, const DrawArgs& A) {
  return o.temperature != 0.0 && !o.by_k && (o.by_p || (o.by_min && A.rows < ROWS_FULL)) && !alone(A);
}
// min-p's border: the least fp32 value that is not below max z + T ln(min_p).
__device__ __forceinline__ float min_p_border(const RowOpts& o, float zmax) {
  const double lowest = (double)zmax + o.temperature * log(fmin(o.min_p, 1.0));
  const float t = (float)lowest;
  return (double)t < lowest ? of_key(key_of(t) + 1) : t;
}
// Part p of a row's segments: a run of them.
__device__ __forceinline__ int part_start(int p, int segs, int parts) { return (int)((int64_t)p * segs / parts); }

// z that many octaves of weight below the largest, a little lower for what was rounded on
// the way.
__device__ __forceinline__ float octaves_below(float zmax, float octaves, double c) {
  const float t = (float)((double)zmax - ((double)octaves + 2e-3) / c);
  return t <= -3.4e38f ? -INFINITY : of_key(key_of(t) - 2);
}

// What the scan knows of a row, put together by a workgroup of N threads.  No barrier stands
// behind the last reads of `red`: only what begins with one may write it next.
struct Row {
  float zmax;
  double total;
  bool good;                          // whether it has an answer
};
template <int N>
__device__ __forceinline__ Row read_row(const DrawArgs& A, const Exp2& exp2, int r, int segs, const RowOpts& o, double* red,
                                        int* redi) {
  const float* top = A.seg_m + (int64_t)r * segs;
  const double* sum = A.seg_s + (int64_t)r * segs;
  const int tid = threadIdx.x;
  int most = rank_of(-INFINITY);
#pragma unroll 2
  for (int i = tid; i < segs; i += N) most = max(most, rank_of(top[i]));
  Row w;
  w.zmax = of_rank(-group_min<N>(-most, redi));
  w.total = 0.0;
  w.good = w.zmax > -INFINITY && w.zmax < INFINITY && usable(o);     // NaN too is none
  if (!w.good) return w;
  double part = 0.0;
#pragma unroll 1
  for (int i = tid; i < segs; i += N) part += share_of(exp2, top[i], sum[i], w.zmax, o.c);
  group_prefix<N>(part, red, &w.total);
  return w;
}

// The least z that top-p can keep (see above): every wave of the workgroup tries another
// distance from the top, in octaves, and what is left between two of them is tried again.
struct MassMemory {
  float share[MAX_SEGS], down[MAX_SEGS];
  int pass[8];
};
template <int N>
__device__ __forceinline__ float least_of_mass(const DrawArgs& A, const Exp2& exp2, int r, int segs, const RowOpts& o, const Row& w,
                                               MassMemory& M) {
  constexpr int W = N / 64;
  static_assert(W == 4 || W == 8, "a flag a wave, and about 700 steps in all");
  const float* top = A.seg_m + (int64_t)r * segs;
  const double* sum = A.seg_s + (int64_t)r * segs;
  const float cf = bin_factor(o.c);
  const double spare = (1.0 - fmax(o.top_p, 0.0)) * w.total * (1.0 - 1e-5);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float lo = 0.f, hi = FIXED_OCTAVES;
#pragma unroll 1
  for (int i = tid; i < segs; i += N) {
    M.share[i] = (float)share_of(exp2, top[i], sum[i], w.zmax, o.c);
    M.down[i] = (w.zmax - top[i]) * cf;
  }
#pragma unroll 1
  for (int round = 0; round < (W == 4 ? 4 : 3); ++round) {
    __syncthreads();
    const float step = (hi - lo) * (1.f / (W + 1)), y = lo + step * (float)(wave + 1);
    const float cap = (float)SEG * __builtin_amdgcn_exp2f(-y);
    double below = 0.0;
#pragma unroll 2
    for (int i = lane; i < segs; i += 64) below += M.down[i] <= y ? fminf(M.share[i], cap) : M.share[i];
    below = lane_of(wave_prefix(below), 63);
    if (lane == 0) M.pass[wave] = below <= spare;
    __syncthreads();
    int first = W;
#pragma unroll
    for (int i = W - 1; i >= 0; --i) first = M.pass[i] ? i : first;
    if (first < W) hi = lo + step * (float)(first + 1);
    lo += step * (float)first;
  }
  return octaves_below(w.zmax, hi, o.c);
}

// The least z that top-k can keep: k values reach it of those that `each` gives a workgroup
// of N threads, maxima or the tokens' own.  They are counted by their distance from the top.
template <int N, typename Each>
__device__ __forceinline__ float least_of(const Each& each, int k, float zmax, double c, uint32_t (&count)[STEPS], int* red) {
  constexpr int PER = STEPS > N ? STEPS / N : 1;
  const int tid = threadIdx.x;
  const float per = bin_factor(c) * (STEPS / FIXED_OCTAVES);
  for (int i = tid; i < STEPS; i += N) count[i] = 0;
  __syncthreads();
  each([&](float z) {
    const float step = (zmax - z) * per;
    if (step < (float)STEPS) atomicAdd(&count[(int)step], 1u);
  });
  __syncthreads();
  uint32_t sum = 0, all;
  if (tid * PER < STEPS)
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += count[tid * PER + i];
  sum = group_prefix<N>(sum, (uint32_t*)red, &all);
  int hit = STEPS - 1;
#pragma unroll
  for (int i = PER - 1; i >= 0; --i)
    if (tid * PER < STEPS) {
      if (sum >= (uint32_t)k) hit = tid * PER + i;
      sum -= count[tid * PER + i];
    }
  return octaves_below(zmax, (float)(group_min<N>(hit, red) + 1) * (FIXED_OCTAVES / STEPS), c);
}

// By one wave: the first of n entries, a lane each in turn, at whose end the running sum of
// f(entry), `before` in front of them, passes `want`, and the sum in front of it.  Where
// roundings next to u = 1 leave none: the last that has a weight, and nothing that its
// tokens could pass.
template <typename V, typename F>
__device__ __forceinline__ int entry_at(int n, F f, double& want, V& before) {
  const int lane = threadIdx.x & 63;
  int last = 0;
#pragma unroll 1
  for (int base = 0; base < n; base += 64) {
    const V w = base + lane < n ? f(base + lane) : 0;
    const V end = wave_prefix(w) + before;
    const uint64_t past = __ballot(w > 0 && (double)end > want), some = __ballot(w > 0);
    if (past) {
      const int at = first_lane(past);
      before = lane_of(end - w, at);
      return base + at;
    }
    if (some) last = base + last_lane(some);
    before = lane_of(end, 63);
  }
  want = INFINITY;
  return last;
}

// Where f of a row's tokens can be had from: its logits.
template <typename T, bool VEC>
struct Logits {
  const T* z;
  int vocab;
  float zmax;
  double c;
  const Exp2& exp2;

  __device__ __forceinline__ double weight(float x) const { return x == -INFINITY ? 0.0 : weight_of(exp2, x, zmax, c); }
  __device__ __forceinline__ u64 fixed(float x) const { return x == -INFINITY ? 0 : fixed_of(weight_of(exp2, x, zmax, c)); }
  // f(its tokens' z, 8 a lane, the first's id) for the strips i0 .. i1 - 1 that have a token
  // of t0 or more, by their maxima top_of: eight strips of eight lanes each at a time, the
  // next eight on their way.  Called by N threads, whose waves take up to 64 strips in turn.
  template <int N, typename F>
  __device__ __forceinline__ void strips(const float* top_of, float t0, int i0, int i1, F f) const {
    constexpr int W = N / 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int share = min(max((i1 - i0 + 8 * W - 1) / (8 * W) * 8, 8), 64);
    int base = i0 + share * wave;
    float top = lane < share && base + lane < i1 ? top_of[base + lane] : -INFINITY;
#pragma unroll 1
    for (; base < i1; base += share * W) {
      const bool on = top >= t0 && top > -INFINITY;
      const int next = base + share * W + lane;
      if (lane < share && next < i1) top = top_of[next];
      else top = -INFINITY;
      const uint64_t mask = __ballot(on);
      const int found = __popcll(mask), in_front = __popcll(mask & ((1ull << lane) - 1));
      // lane j has the number of the j-th of them
      const int order = __builtin_amdgcn_ds_permute(4 * (on ? in_front : found + lane - in_front), lane);
      auto fetch = [&](Eight<T, VEC>& v, int& first, int a) {
        const int k = a + (lane >> 3), strip = base + __builtin_amdgcn_ds_bpermute(4 * k, order);
        first = k < found ? strip * STRIP + 8 * (lane & 7) : vocab;
        v.load(z, first, vocab);
      };
      Eight<T, VEC> v, after;
      int first, first_after;
      if (found) fetch(v, first, 0);
#pragma unroll 1
      for (int a = 0; a < found; a += 8) {
        fetch(after, first_after, a + 8);
        f(v, first);
        v = after;
        first = first_after;
      }
    }
  }
  // f(z, id) for their tokens of t0 or more.  DENSE: most of them are.
  template <int N, bool DENSE, typename F>
  __device__ __forceinline__ void tokens(const float* top_of, float t0, int i0, int i1, F f) const {
    strips<N>(top_of, t0, i0, i1, [&](const Eight<T, VEC>& v, int first) {
      if constexpr (DENSE) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (v[e] >= t0 && v[e] > -INFINITY) f(v[e], first + e);   // tokens past the vocabulary are -inf
      } else {
#pragma unroll 1
        for (uint32_t hits = v.from(t0); hits; hits &= hits - 1) {
          const int at = __ffs((int)hits) - 1;
          f(v.at(at), first + at);
        }
      }
    });
  }
  // By a workgroup of N threads: the token of segment s at which the running sum of
  // weigh(z, id), `before` in front of the segment, passes `want`; the last with a weight
  // where none does.  sums: [STRIPS] in shared memory.
  template <int N, typename V, typename W>
  __device__ __forceinline__ int token_at(int s, V before, double want, W weigh, V* sums, float& at_z) const {
    const int lane = threadIdx.x & 63;
    float x;
    int id;
    auto end_of = [&](int strip, V& w) {
      id = s * SEG + strip * STRIP + lane;
      x = id < vocab ? ld_f32<T>(z + id) : -INFINITY;
      w = id < vocab ? weigh(x, id) : 0;
      return wave_prefix(w);
    };
    V w;
    __syncthreads();
#pragma unroll 1
    for (int j = threadIdx.x >> 6; j < STRIPS; j += N / 64) {
      const V end = end_of(j, w);
      if (lane == 63) sums[j] = end;
    }
    __syncthreads();
    const int at = entry_at(STRIPS, [&](int j) { return sums[j]; }, want, before);
    const V end = end_of(at, w) + before;
    const uint64_t past = __ballot(w > 0 && (double)end > want), some = __ballot(w > 0);
    const int from = past ? first_lane(past) : last_lane(some | 1);
    at_z = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), from));
    return __builtin_amdgcn_readlane(id, from);
  }
};

__device__ __forceinline__ double given_u(const DrawArgs& A, int r) {
  return A.u64 ? ((const double*)A.u)[r] : (double)((const float*)A.u)[r];
}
__device__ __forceinline__ void no_answer(const DrawArgs& A, int r) {
  A.token[r] = -1;
  A.logprob[r] = A.kept[r] = __uint_as_float(0x7FC00000u);
}
// By two threads, the first of them and another of its wave: a logarithm each.
__device__ __forceinline__ void answer(const DrawArgs& A, int r, bool first, int id, float z, float zmax, double c, double total,
                                       double kept) {
  const float lp = (float)(((double)z - (double)zmax) * c * 0.6931471805599453 - log(first ? total : kept));
  if (first) {
    A.token[r] = id;
    A.logprob[r] = lp;
  } else {
    A.kept[r] = lp;
  }
}

// By a workgroup of N threads: a row of which nothing is cut, or all but the first of the
// largest (T = 0).
template <int N>
struct PlainMemory {
  double red[N / 64], before, sums[STRIPS];
  int redi[N / 64];
};
template <int N, typename T, bool VEC>
__device__ __forceinline__ void draw_plain(const DrawArgs& A, PlainMemory<N>& P, int r, int segs, const Row& w,
                                           const Logits<T, VEC>& z, const RowOpts& o, double u) {
  const float* top = A.seg_m + (int64_t)r * segs;
  const double* sum = A.seg_s + (int64_t)r * segs;
  const int tid = threadIdx.x;
  const bool greedy = o.temperature == 0.0;
  double want = greedy ? 0.0 : u * w.total, before = 0.0;
  int at = INT32_MAX, last = 0;
#pragma unroll 1
  for (int base = 0; base < segs && at == INT32_MAX; base += N) {
    const int i = base + tid;
    double x = 0.0, all;
    if (i < segs) x = greedy ? (double)(top[i] == w.zmax) : share_of(z.exp2, top[i], sum[i], w.zmax, o.c);
    const double end = group_prefix<N>(x, P.red, &all) + before;
    at = group_min<N>(x > 0.0 && end > want ? i : INT32_MAX, P.redi);
    if (at == i) P.before = end - x;
    last = max(last, -group_min<N>(x > 0.0 ? -i : 0, P.redi));
    before += all;
  }
  __syncthreads();
  if (at == INT32_MAX) {              // roundings next to u = 1
    at = last;
    want = INFINITY;
  } else {
    before = P.before;
  }
  if (greedy) before = 0.0;
  float at_z;
  const int id = z.template token_at<N>(
      at, before, want, [&](float x, int) { return greedy ? (double)(x == w.zmax) : z.weight(x); }, P.sums, at_z);
  if (tid < 2) answer(A, r, tid == 0, id, at_z, w.zmax, o.c, w.total, greedy ? 1.0 : w.total);
}

template <typename T, bool VEC>
__global__ __launch_bounds__(PART) void k_draw_plain(DrawArgs A, int segs) {
  __shared__ PlainMemory<PART> P;
  const int r = blockIdx.x;
  const RowOpts o = row_opts(A, r);
  const double u = given_u(A, r);
  const Exp2 exp2;
  const Row w = read_row<PART>(A, exp2, r, segs, o, P.red, P.redi);
  if (!w.good || !(u >= 0.0 && u < 1.0)) {
    if (threadIdx.x == 0) no_answer(A, r);
    return;
  }
  draw_plain<PART>(A, P, r, segs, w, Logits<T, VEC>{(const T*)A.logits + r * A.row, A.vocab, w.zmax, o.c, exp2}, o, u);
}

// ---------------------------------------------------------------- bins, collect
template <typename T, bool VEC>
__global__ __launch_bounds__(PART) void k_draw_bins(DrawArgs A, int segs, int parts) {
  __shared__ union {
    u64 mass[BINS];
    MassMemory least;
  } L;
  __shared__ double red[PART / 64];
  __shared__ int redi[PART / 64];
  const int r = blockIdx.x / parts, part = blockIdx.x - r * parts, tid = threadIdx.x;
  const RowOpts o = row_opts(A, r);
  if (!by_bins(o, A)) return;
  const Exp2 exp2;
  const Row w = read_row<PART>(A, exp2, r, segs, o, red, redi);
  float t0 = 0.f;
  if (w.good) {
    t0 = o.by_p ? least_of_mass<PART>(A, exp2, r, segs, o, w, L.least) : octaves_below(w.zmax, FIXED_OCTAVES, o.c);
    if (o.by_min) t0 = fmaxf(t0, min_p_border(o, w.zmax));
  }
  if (part == 0 && tid == 0) A.info[r] = DrawRow{w.total, w.zmax, t0, w.good, 0, BINS, 0};
  if (!w.good) return;
  __syncthreads();
  for (int i = tid; i < BINS; i += PART) L.mass[i] = 0;
  __syncthreads();
  const float per = bins_per_logit(w.zmax, t0, bin_factor(o.c));
  const Logits<T, VEC> z{(const T*)A.logits + r * A.row, A.vocab, w.zmax, o.c, exp2};
  z.template tokens<PART, true>(A.strip_m + (int64_t)r * segs * STRIPS, t0, part_start(part, segs, parts) * STRIPS,
                                part_start(part + 1, segs, parts) * STRIPS,
                                [&](float x, int) { atomicAdd(&L.mass[bin_of(x, w.zmax, per)], z.fixed(x)); });
  __syncthreads();
  u64* bins = A.part_bins + (int64_t)blockIdx.x * BINS;
#pragma unroll 1
  for (int i = tid; i < BINS; i += PART) {
    const u64 m = L.mass[i];
    bins[i] = m;
    if (m) atomicAdd(&A.bins[(int64_t)r * BINS + i], m);
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(PART) void k_draw_collect(DrawArgs A, int segs, int parts) {
  __shared__ u64 red[8], list[LIST];
  __shared__ int redi[8], n_list, at;
  const int r = blockIdx.x / parts, part = blockIdx.x - r * parts, tid = threadIdx.x;
  const RowOpts o = row_opts(A, r);
  if (!by_bins(o, A)) return;
  const DrawRow info = A.info[r];
  if (!info.good) return;
  if (tid == 0) n_list = 0;
  constexpr int PER = BINS / PART;
  u64 mine[PER], own[PER], all, kept = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    mine[i] = A.bins[(int64_t)r * BINS + tid * PER + i];
    own[i] = A.part_bins[(int64_t)blockIdx.x * BINS + tid * PER + i];
  }
  const double limit = mass_limit(o, info.total * FIXED_ONE);
  u64 sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) sum += mine[i];
  u64 end = group_prefix<PART>(sum, red, &all);
  int hit = BINS;
  u64 before = end;
#pragma unroll
  for (int i = PER - 1; i >= 0; --i) {
    if (o.by_p && mine[i] && (double)end >= limit) {
      hit = tid * PER + i;
      before = end - mine[i];
    }
    end -= mine[i];
  }
  const int border = group_min<PART>(hit, redi);   // the bin in which top-p's border lies
  if (part == 0 && hit == border && border < BINS) {
    A.info[r].bin = border;
    A.info[r].above = before;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (tid * PER + i < border) kept += own[i];       // what the part keeps above it
  group_prefix<PART>(kept, red, &all);
  if (tid == 0) A.part_kept[blockIdx.x] = all;
  if (border == BINS) return;
  const float per = bins_per_logit(info.zmax, info.t0, bin_factor(o.c));
  const Exp2 exp2;
  const Logits<T, VEC> z{(const T*)A.logits + r * A.row, A.vocab, info.zmax, o.c, exp2};
  z.template tokens<PART, true>(A.strip_m + (int64_t)r * segs * STRIPS, info.t0, part_start(part, segs, parts) * STRIPS,
                                part_start(part + 1, segs, parts) * STRIPS, [&](float x, int id) {
                                  if (bin_of(x, info.zmax, per) != border) return;
                                  const int k = atomicAdd(&n_list, 1);
                                  if (k < LIST) list[k] = Places<T>::of(x, id);
                                });
  __syncthreads();
  const int n = n_list;
  if (n == 0) return;
  if (tid == 0) at = atomicAdd(&A.info[r].listed, n);
  __syncthreads();
  for (int i = tid; i < min(n, LIST); i += PART)
    if (at + i < LIST) A.list[(int64_t)r * LIST + at + i] = list[i];
}

// ---------------------------------------------------------------- pick
template <int N>
struct CutMemory {
  static constexpr int FEW = 128;       // tokens that are compared with one another (256: 22 us in place of 18)
  struct Token { u64 place, weight; };
  union {
    struct { u64 mass[BINS]; uint32_t count[BINS]; } bin;
    u64 seg[MAX_SEGS];                // kept weight of each segment
    uint32_t steps[STEPS];
    PlainMemory<N> plain;
    MassMemory least;
  };
  u64 list[LIST];                     // places of the tokens that can be kept
  Token few[FEW];
  u64 before[FEW];
  int rank[FEW];
  u64 red[N / 64], sums[STRIPS], found, mass, rank0, lo, hi;
  // the row's sum: of its own, since what comes next fills the union while other waves may
  // still be reading it
  double total[N / 64];
  int redi[N / 64], n_list, n_few;
};

// The first n <= FEW tokens of C.few, a thread each and the rest of the workgroup to share
// their comparisons: how many of them come before the thread's, and what those weigh.
template <int N>
__device__ __forceinline__ void compare(CutMemory<N>& C, int n, int& rank, u64& before) {
  constexpr int FEW = CutMemory<N>::FEW;
  const int tid = threadIdx.x;
  const int room = n <= 64 ? 64 : 128, groups = N / room, mine = tid % room, per = (n + groups - 1) / groups;
  static_assert(FEW == 128 && FEW <= N, "a thread has one token at most");
  if (tid < n) {
    C.before[tid] = 0;
    C.rank[tid] = 0;
  }
  __syncthreads();
  int k = 0;
  u64 w = 0;
  if (mine < n) {
    const u64 p = C.few[mine].place;
    const int end = min(n, (tid / room + 1) * per);
#pragma unroll 4
    for (int j = tid / room * per; j < end; ++j) {
      const bool in_front = C.few[j].place > p;
      k += in_front;
      w += in_front ? C.few[j].weight : 0;
    }
    if (k) {
      atomicAdd(&C.rank[mine], k);
      atomicAdd(&C.before[mine], w);
    }
  }
  __syncthreads();
  rank = tid < n ? C.rank[tid] : 0;
  before = tid < n ? C.before[tid] : 0;
}

// The border of top-k (by rank: fewer than `limit` tokens come before) or top-p (less
// than `limit` of weight does) among the tokens that `each` gives, n of them, mass0 of
// weight in front of them, none outside the places lo .. hi: the place of the last that is
// kept, 0 if all of them are; mass: the weight up to it.  Windows of places, ever finer by
// 1024, until what is left can be compared.
template <typename P, int N, typename R, typename Each>
__device__ __forceinline__ u64 find_border(const R& row, CutMemory<N>& C, const Each& each, int n, bool by_rank, double limit,
                                           u64 lo, u64 hi, u64 mass0, u64* mass) {
  constexpr int FEW = CutMemory<N>::FEW, PER = BINS / N;
  const int tid = threadIdx.x;
  u64 rank0 = 0;                      // before the window
  int inside = n;
  auto reaches = [&](u64 rank, u64 weight) { return by_rank ? (double)rank >= limit : (double)weight >= limit; };
#pragma unroll 1
  while (inside > FEW) {              // places differ: at the latest a window of one has one token
    __syncthreads();
    for (int i = tid; i < BINS; i += N) { C.bin.mass[i] = 0; C.bin.count[i] = 0; }
    __syncthreads();
    const int shift = max(54 - __clzll((long long)(hi - lo | 1)), 0);   // (hi - lo) >> shift is below 1024
    each([&](float x, int id) {
      const u64 p = P::of(x, id);
      if (p < lo || p > hi) return;
      const int d = BINS - 1 - (int)((p - lo) >> shift);
      atomicAdd(&C.bin.mass[d], row.fixed(x));
      atomicAdd(&C.bin.count[d], 1u);
    });
    __syncthreads();
    // the first digit whose end reaches the limit
    u64 m = 0, rank = 0, all_m, all_n;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      m += C.bin.mass[tid * PER + i];
      rank += C.bin.count[tid * PER + i];
    }
    m = group_prefix<N>(m, C.red, &all_m) + mass0;
    rank = group_prefix<N>(rank, C.red, &all_n) + rank0;
    int hit = INT32_MAX;
    u64 hit_m = 0, hit_n = 0;
#pragma unroll
    for (int i = PER - 1; i >= 0; --i) {
      const u64 w = C.bin.mass[tid * PER + i], k = C.bin.count[tid * PER + i];
      if (k && reaches(rank, m)) {
        hit = tid * PER + i;
        hit_m = m - w;
        hit_n = rank - k;
      }
      m -= w;
      rank -= k;
    }
    const int d = group_min<N>(hit, C.redi);
    if (d == INT32_MAX) {             // the limit lies behind the last token
      *mass = mass0 + all_m;
      return 0;
    }
    if (hit == d) {
      C.mass = hit_m;
      C.rank0 = hit_n;
    }
    __syncthreads();
    mass0 = C.mass;
    rank0 = C.rank0;
    inside = (int)min(C.bin.count[d], (uint32_t)FEW + 1);
    lo += (u64)(BINS - 1 - d) << shift;
    hi = min(hi, lo + ((1ull << shift) - 1));
  }
  __syncthreads();
  if (tid == 0) C.n_few = 0;
  __syncthreads();
  each([&](float x, int id) {
    const u64 p = P::of(x, id);
    if (p >= lo && p <= hi) C.few[atomicAdd(&C.n_few, 1)] = {p, row.fixed(x)};
  });
  if (tid == 0) C.found = 0;
  __syncthreads();
  const int k = C.n_few;
  int rank;
  u64 before;
  compare(C, k, rank, before);
  const u64 p = tid < k ? C.few[tid].place : 0, w = tid < k ? C.few[tid].weight : 0;
  const u64 end = mass0 + before + w;
  if (tid < k && !reaches(rank0 + rank, mass0 + before) && reaches(rank0 + rank + 1, end)) {
    C.found = p;
    C.mass = end;
  }
  if (tid < k && rank == k - 1) C.hi = end;   // the limit may lie behind the last token
  __syncthreads();
  const u64 found = C.found;
  *mass = found ? C.mass : k ? C.hi : mass0;
  return found;
}

template <typename T, bool VEC, int N>
__global__ __launch_bounds__(N) void k_draw_pick(DrawArgs A, int segs, int parts) {
  typedef Places<T> P;
  __shared__ CutMemory<N> C;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const RowOpts o = row_opts(A, r);
  const double u = given_u(A, r);
  const bool binned = by_bins(o, A);
  const Exp2 exp2;
  DrawRow info{};
  Row w;
  float t0 = 0.f;                     // no token below it is kept
  if (binned) {
    info = A.info[r];
    t0 = info.t0;
    w = Row{info.zmax, info.total, info.good != 0};
  } else {
    w = read_row<N>(A, exp2, r, segs, o, C.total, C.redi);
  }
  if (!w.good || !(u >= 0.0 && u < 1.0)) {
    if (tid == 0) no_answer(A, r);
    return;
  }
  const Logits<T, VEC> z{(const T*)A.logits + r * A.row, A.vocab, w.zmax, o.c, exp2};
  if (o.temperature == 0.0 || !(o.by_k || o.by_p || o.by_min)) {   // nothing is cut here
    draw_plain<N>(A, C.plain, r, segs, w, z, o, u);
    return;
  }
  const float min_z = o.by_min ? min_p_border(o, w.zmax) : -INFINITY;
  u64 border = o.by_min ? P::from(min_z) : 0;
  const bool whole_list = binned && info.listed <= LIST;   // the border's bin is listed, the rest summed
  const int n_strips = segs * STRIPS;
  const float* const strip_m = A.strip_m + (int64_t)r * n_strips;
  bool known = !binned && !o.by_k && !o.by_p;              // the border: no list is needed
  const bool own_bins = !binned && !o.by_k && o.by_p && A.vocab > OWN_BINS;
  int bin = BINS;                                          // of those the one in which the border lies
  float per = 0.f;
  u64 above = whole_list ? info.above : 0;
  if (o.by_k) {
    // segments' maxima tell where there are twice as many, else strips', else the tokens
    const float far = octaves_below(w.zmax, FIXED_OCTAVES, o.c);
    const bool coarse = 2 * o.top_k <= segs;
    const int n = coarse ? segs : n_strips;
    const float* const top = coarse ? A.seg_m + (int64_t)r * segs : strip_m;
    t0 = least_of<N>(
        [&](auto f) {
          if (2 * o.top_k <= n) {
#pragma unroll 4
            for (int i = tid; i < n; i += N) f(top[i]);
          } else {
            z.template tokens<N, true>(strip_m, far, 0, n_strips, [&](float x, int) { f(x); });
          }
        },
        o.top_k, w.zmax, o.c, C.steps, C.redi);
  } else if (own_bins) {
    t0 = least_of_mass<N>(A, exp2, r, segs, o, w, C.least);
  } else if (!binned) {
    t0 = octaves_below(w.zmax, FIXED_OCTAVES, o.c);
  }
  if (!binned && !(o.by_k && o.by_p)) t0 = fmaxf(t0, min_z);   // top-p takes its share of all the k
  if (own_bins) {
    constexpr int PER = BINS / N;
    per = bins_per_logit(w.zmax, t0, bin_factor(o.c));
    __syncthreads();
    for (int i = tid; i < BINS; i += N) C.bin.mass[i] = 0;
    __syncthreads();
    z.template tokens<N, true>(strip_m, t0, 0, n_strips,
                               [&](float x, int) { atomicAdd(&C.bin.mass[bin_of(x, w.zmax, per)], z.fixed(x)); });
    __syncthreads();
    u64 mine[PER], sum = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += mine[i] = C.bin.mass[tid * PER + i];
    u64 end = group_prefix<N>(sum, C.red, &all);
    int hit = BINS;
    u64 front = 0;
#pragma unroll
    for (int i = PER - 1; i >= 0; --i) {
      if (mine[i] && (double)end >= mass_limit(o, w.total * FIXED_ONE)) {
        hit = tid * PER + i;
        front = end - mine[i];
      }
      end -= mine[i];
    }
    bin = group_min<N>(hit, C.redi);
    known = bin == BINS;
    if (hit == bin && !known) C.mass = front;
    __syncthreads();
    if (!known) above = C.mass;
  }
  if (tid == 0) {
    C.n_list = whole_list ? info.listed : known ? LIST + 1 : 0;
    C.lo = ~0ull;
    C.hi = 0;
  }
  __syncthreads();
  if (whole_list) {
    for (int i = tid; i < info.listed; i += N) C.list[i] = A.list[(int64_t)r * LIST + i];
  } else if (!known) {
    z.template strips<N>(strip_m, t0, 0, n_strips, [&](const Eight<T, VEC>& v, int first) {
      uint32_t hits = v.from(t0);
      if (own_bins)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (bin_of(v[e], w.zmax, per) != bin) hits &= ~(1u << e);
      const int mine = __popc(hits), end = wave_prefix(mine);
      int at = 0;
      if (lane == 63) at = atomicAdd(&C.n_list, end);
      at = __builtin_amdgcn_readlane(at, 63) + end - mine;
#pragma unroll 1
      for (; hits; hits &= hits - 1, ++at) {
        const int e = __ffs((int)hits) - 1;
        if (at < LIST) C.list[at] = P::of(v.at(e), first + e);
      }
    });
  }
  __syncthreads();
  const int n_list = C.n_list;

  // Few of all that can be kept: a thread each, compared with one another and drawn from by
  // their ids.
  if (!whole_list && !own_bins && n_list <= CutMemory<N>::FEW) {
    const bool is = tid < n_list;
    const u64 p = is ? C.list[tid] : 0, mine = is ? z.fixed(P::z(p)) : 0;
    const int id = P::id(p);
    if (is) C.few[tid] = {p, mine};
    __syncthreads();
    int rank;
    u64 before, all;
    compare(C, n_list, rank, before);
    bool in = is && (!o.by_k || rank < o.top_k);
    if (o.by_p) {
      double share = w.total * FIXED_ONE;
      if (o.by_k) {
        group_prefix<N>(in ? mine : (u64)0, C.red, &all);
        share = (double)all;
      }
      in = in && (double)before < mass_limit(o, share);
    }
    in = in && p >= border;
    group_prefix<N>(in ? mine : (u64)0, C.red, &all);
    const double want = u * (double)all;
    // again by id, the lowest first, of what is kept: the first whose end passes
    if (is) C.few[tid] = {(u64)(0xFFFFFFFFu - id), in ? mine : 0};
    __syncthreads();
    compare(C, n_list, rank, before);
    const bool can = in && mine > 0;
    const int past = group_min<N>(can && (double)(before + mine) > want ? id : INT32_MAX, C.redi);
    // roundings next to u = 1: the highest with a weight
    int hit = past;
    if (past == INT32_MAX) hit = -group_min<N>(can ? -id : 0, C.redi);
    if (can && id == hit) C.found = p;
    __syncthreads();
    if (tid < 2) answer(A, r, tid == 0, hit, P::z(C.found), w.zmax, o.c, w.total, (double)all / FIXED_ONE);
    return;
  }

  auto each = [&](auto f) {
    if (n_list <= LIST) {
      for (int i = tid; i < n_list; i += N) f(P::z(C.list[i]), P::id(C.list[i]));
    } else {
      z.template tokens<N, false>(strip_m, t0, 0, n_strips, f);
    }
  };
  u64 lo = P::of(t0, (1 << ID_BITS) - 1), hi = P::of(w.zmax, 0);
  if (n_list <= LIST) {               // no wider than the list is
    u64 least = ~0ull, most = 0;
    for (int i = tid; i < n_list; i += N) {
      least = min(least, C.list[i]);
      most = max(most, C.list[i]);
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) {
      least = min(least, __shfl_xor(least, x, 64));
      most = max(most, __shfl_xor(most, x, 64));
    }
    if (lane == 0 && most) {
      atomicMin(&C.lo, least);
      atomicMax(&C.hi, most);
    }
    __syncthreads();
    lo = C.lo;
    hi = C.hi;
  }
  double share = w.total * FIXED_ONE;
#pragma unroll 1
  for (int rule = 0; rule < 2; ++rule) {
    if (rule == 0 ? !o.by_k : !o.by_p || known || (whole_list && info.bin == BINS)) continue;
    u64 mass;
    border = max(border, find_border<P>(z, C, each, n_list, rule == 0, rule == 0 ? (double)o.top_k : mass_limit(o, share), lo, hi,
                                        n_list <= LIST ? above : 0, &mass));
    share = (double)mass;
  }
  // What is kept of each segment or, where the histogram knows the parts', of each part
  // and then of that part's segments.
  __syncthreads();
  int s0 = 0, s1 = segs;
  u64 before = 0, kept = 0;
  double want = 0.0;
  if (whole_list) {
    for (int i = tid; i < parts; i += N) C.seg[i] = A.part_kept[(int64_t)r * parts + i];
    __syncthreads();
    for (int i = tid; i < n_list; i += N)
      if (C.list[i] >= border) {
        const int s = P::id(C.list[i]) / SEG;
        int p = (int)((int64_t)s * parts / segs);
        while (part_start(p + 1, segs, parts) <= s) ++p;
        atomicAdd(&C.seg[p], z.fixed(P::z(C.list[i])));
      }
    __syncthreads();
    for (int i = lane; i < parts; i += 64) kept += C.seg[i];
    kept = lane_of(wave_prefix(kept), 63);
    want = u * (double)kept;
    const int p = entry_at(parts, [&](int i) { return C.seg[i]; }, want, before);
    s0 = part_start(p, segs, parts);
    s1 = part_start(p + 1, segs, parts);
    __syncthreads();
  }
  for (int i = s0 + tid; i < s1; i += N) C.seg[i] = 0;
  __syncthreads();
  if (!whole_list && !own_bins && n_list <= LIST) {
    each([&](float x, int id) {
      if (P::of(x, id) >= border) atomicAdd(&C.seg[id / SEG], z.fixed(x));
    });
  } else {                            // a strip's tokens add up within its lanes
    z.template strips<N>(strip_m, t0, s0 * STRIPS, s1 * STRIPS, [&](const Eight<T, VEC>& v, int first) {
      u64 sum = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (v[e] >= t0 && P::of(v[e], first + e) >= border) sum += z.fixed(v[e]);
      sum += shifted<0x111, 0xF>(sum);   // to the last of the eight lanes
      sum += shifted<0x112, 0xF>(sum);
      sum += shifted<0x114, 0xF>(sum);
      if ((lane & 7) == 7 && sum) atomicAdd(&C.seg[first / SEG], sum);
    });
  }
  __syncthreads();
  if (!whole_list) {
    for (int i = lane; i < segs; i += 64) kept += C.seg[i];
    kept = lane_of(wave_prefix(kept), 63);
    want = u * (double)kept;
  }
  const int at = s0 + entry_at(s1 - s0, [&](int i) { return C.seg[s0 + i]; }, want, before);
  float at_z;
  const int id = z.template token_at<N>(
      at, before, want, [&](float x, int i) { return P::of(x, i) >= border ? z.fixed(x) : (u64)0; }, C.sums, at_z);
  if (tid < 2) answer(A, r, tid == 0, id, at_z, w.zmax, o.c, w.total, (double)kept / FIXED_ONE);
}

int segments(int vocab) { return (vocab + SEG - 1) / SEG; }

// Whether rows may be cut, and whether some may go by histogram.
bool may_cut(const DrawArgs& a) {
  return a.top_k_rows || a.top_p_rows || a.min_p_rows || a.top_k > 0 || a.top_p < 1.0 || a.min_p > 0.0;
}
bool may_bin(const DrawArgs& a) {
  return !alone(a) && (a.top_k_rows || a.top_k == 0 || a.top_k >= a.vocab) &&
         (a.top_p_rows || a.top_p < 1.0 || (a.rows < ROWS_FULL && (a.min_p_rows || a.min_p > 0.0)));
}

// Parts of a row in the histogram: enough to fill the chip, of eight segments at least,
// and few enough to go through one again in the pick.
int parts_of(const DrawArgs& a) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::max<int64_t>(1024 / a.rows, 4), (segments(a.vocab) + 7) / 8));
}

// Where the parts of the scratch are.
struct Scratch {
  int64_t seg_s, part_bins, part_kept, bins, list, info, seg_m, strip_m, end;
};
Scratch scratch_of(const DrawArgs& a) {
  const int64_t rows = a.rows, n = rows * segments(a.vocab), binned = may_bin(a) ? rows : 0, parts = binned * parts_of(a);
  Scratch s;
  s.seg_s = 0;
  s.part_bins = s.seg_s + 8 * n;
  s.part_kept = s.part_bins + 8 * parts * BINS;
  s.bins = s.part_kept + 8 * parts;
  s.list = s.bins + 8 * binned * BINS;
  s.info = s.list + 8 * binned * LIST;
  s.seg_m = s.info + (int64_t)sizeof(DrawRow) * binned;
  s.strip_m = s.seg_m + 4 * n;
  s.end = (s.strip_m + (may_cut(a) ? 4 * STRIPS * n : 0) + 15) / 16 * 16;
  return s;
}

template <typename T, bool VEC>
hipError_t run(const DrawArgs& a, hipStream_t st) {
  const int segs = segments(a.vocab), parts = parts_of(a);
  const unsigned per_row = (unsigned)(segs + 1) / 2;
  const int64_t items = (int64_t)a.rows * per_row;
  // the scan does not run where a launch behind it would be one of 2^32 threads
  const int64_t threads = std::max<int64_t>((int64_t)a.rows * (may_cut(a) ? PICK : PART), a.bins ? (int64_t)a.rows * parts * PART : 0);
  if (items > INT32_MAX / 2 || threads >> 32) return hipErrorInvalidValue;
  const int64_t per = std::max<int64_t>(1, items / SCAN_FILL), waves = (items + per - 1) / per;
  const dim3 grid((unsigned)((waves + SCAN_WAVES - 1) / SCAN_WAVES)), scan(64 * SCAN_WAVES);
  const dim3 part((unsigned)(a.rows * parts)), rows(a.rows);
  const unsigned n = (unsigned)items, each = (unsigned)per;
  hipError_t e;
  if (!may_cut(a)) {
    if ((e = kv8_launch(k_draw_scan<T, VEC, false>, grid, scan, st, a, segs, per_row, n, each)) != hipSuccess) return e;
    return kv8_launch(k_draw_plain<T, VEC>, rows, dim3(PART), st, a, segs);
  }
  if ((e = kv8_launch(k_draw_scan<T, VEC, true>, grid, scan, st, a, segs, per_row, n, each)) != hipSuccess) return e;
  if (a.bins) {
    if ((e = kv8_launch(k_draw_bins<T, VEC>, part, dim3(PART), st, a, segs, parts)) != hipSuccess) return e;
    if ((e = kv8_launch(k_draw_collect<T, VEC>, part, dim3(PART), st, a, segs, parts)) != hipSuccess) return e;
  }
  return kv8_launch(k_draw_pick<T, VEC, PICK>, rows, dim3(PICK), st, a, segs, parts);
}

}  // namespace

int64_t draw_scratch_bytes(const DrawArgs& a) { return scratch_of(a).end; }

hipError_t launch_draw(DrawArgs a, void* scratch, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  if (a.vocab < 1 || a.vocab > DRAW_MAX_VOCAB) return hipErrorInvalidValue;
  const Scratch s = scratch_of(a);
  char* p = (char*)scratch;
  a.c = a.temperature == 0.0 ? LOG2E : std::min(LOG2E / a.temperature, 1e300);   // finite: 0 c is 0
  a.seg_s = (double*)(p + s.seg_s);
  a.seg_m = (float*)(p + s.seg_m);
  a.strip_m = (float*)(p + s.strip_m);
  if (may_bin(a)) {
    a.part_bins = (unsigned long long*)(p + s.part_bins);
    a.part_kept = (unsigned long long*)(p + s.part_kept);
    a.bins = (unsigned long long*)(p + s.bins);
    a.list = (unsigned long long*)(p + s.list);
    a.info = (DrawRow*)(p + s.info);
  }
  const bool vec = (uintptr_t)a.logits % 16 == 0 && a.row * (a.dtype == 1 ? 2 : 4) % 16 == 0;
  if (a.dtype == 1) return vec ? run<bf16_t, true>(a, st) : run<bf16_t, false>(a, st);
  return vec ? run<float, true>(a, st) : run<float, false>(a, st);
}
