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
// thousand.  Weights are therefore fp64, by a polynomial of their own (exp2_64, 1e-12):
// 16 instructions a token, which still fit under the bytes of fp32 logits.  Where
// something is cut the weights are whole numbers, w 2^42 to nearest: their sums do not
// depend on any order, so atomics give the same draw on every run.
//
// Launches:
// * scan, a wave four segments of 512 tokens: maximum, and sum of weights with respect to
//   it; maxima of strips of 64.  It streams the logits once.
// * where nothing can be cut: plain, a wave a row.  The segment at which the running sum
//   passes, then the token.
// * only where top-p or min-p may cut a row without top-k: rows (a wave a row: its sum, and
//   the least z that can be kept), bins and collect (some workgroups a row, each a part of
//   it).  The bins add up weights by z; collect finds the bin in which the border of top-p
//   lies, sums what each part keeps above it, and lists the tokens in it.
// * pick, a workgroup a row: the border, then where the running sum passes.
// All after the scan look only at segments that can hold kept tokens:
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
constexpr int SCAN_WAVES = 4;
constexpr int PICK = 256;             // threads of a row's pick
constexpr int PART = 256;             // threads of a part of a row's histogram
constexpr int BINS = 1024;            // of z, 16 an octave of weight
constexpr int LIST = 4096;            // tokens that a row's list holds
constexpr int FEW = 64;               // tokens that a wave compares with one another
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
  __device__ __forceinline__ double operator()(double t) const {
    constexpr double shifter = 6755399441055744.0;            // 1.5 * 2^52: the sum's low bits are t to nearest
    const double s = t + shifter, f = t - (s - shifter);
    double p = __builtin_bit_cast(double, a[0]);
#pragma unroll
    for (int i = 1; i < N; ++i) p = fma(p, f, __builtin_bit_cast(double, a[i]));
    p = fma(p, f, 1.0);
    u32x2_t w = __builtin_bit_cast(u32x2_t, p);               // n into the exponent: of the high word alone
    w[1] += __builtin_bit_cast(u32x2_t, s)[0] << 20;
    return __builtin_bit_cast(double, w);
  }
};
__device__ __forceinline__ double exp2_64(double t) { return Exp2()(t); }
// The weight of z with respect to top (finite, no less): octaves below 1000 count nothing.
__device__ __forceinline__ double weight_of(float z, float top, double c) {
  return exp2_64(fmax(((double)z - (double)top) * c, -1000.0));
}
// w 2^42 to nearest.
__device__ __forceinline__ u64 fixed_of(double w) {
  return __builtin_bit_cast(u64, fma(w, FIXED_ONE, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;   // 2^52 + w 2^42
}

// NaN where either is.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// The wave's sum, in lane 63 alone: lanes past a row's end, and rows without a source, add
// 0; what the middle rows take in twice never gets there.
template <int CTRL>
__device__ __forceinline__ double moved(double v) {
  const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
  return __builtin_bit_cast(double, u32x2_t{(uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[0], CTRL, 0xf, 0xf, true),
                                            (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[1], CTRL, 0xf, 0xf, true)});
}
__device__ __forceinline__ double sum_to_63(double v) {
  v += moved<0x111>(v);               // row_shr 1, 2, 4, 8, then row_bcast 15 and 31
  v += moved<0x112>(v);
  v += moved<0x114>(v);
  v += moved<0x118>(v);
  v += moved<0x142>(v);
  v += moved<0x143>(v);
  return v;
}
__device__ __forceinline__ double from_63(double v) {
  const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
  return __builtin_bit_cast(double, u32x2_t{(uint32_t)__builtin_amdgcn_readlane((int)w[0], 63),
                                            (uint32_t)__builtin_amdgcn_readlane((int)w[1], 63)});
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
__device__ __forceinline__ float max_nan_wave(float z) {
  int v = rank_of(z);
  v = max_moved<0x111>(v);
  v = max_moved<0x112>(v);
  v = max_moved<0x114>(v);
  v = max_moved<0x118>(v);
  v = max_moved<0x142>(v);
  v = max_moved<0x143>(v);
  return of_rank(__builtin_amdgcn_readlane(v, 63));
}
__device__ __forceinline__ float sum_wave(float v) { return (float)from_63(sum_to_63((double)v)); }

template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int i, int n, float (&v)[8]) {
  if (VEC && i + 8 <= n) {
    ld_elems<8, true>(p + i, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = i + e < n ? ld_f32<T>(p + i + e) : -INFINITY;
  }
}

// ---------------------------------------------------------------- scan
// Four segments a wave: their loads are on their way together, and the lane moves of one
// fill the waits of another.
template <typename T, bool VEC, bool CUT>
__global__ __launch_bounds__(64 * SCAN_WAVES) void k_draw_scan(DrawArgs A, int segs, unsigned per_row, unsigned items) {
  constexpr int U = 4;
  const int lane = threadIdx.x & 63;
  const unsigned item = blockIdx.x * SCAN_WAVES + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (item >= items) return;
  const unsigned r = item / per_row;
  const int s0 = (int)(item - r * per_row) * U;
  const T* z = (const T*)A.logits + r * A.row;
  float v[U][8], m[U];
#pragma unroll
  for (int j = 0; j < U; ++j) load8<T, VEC>(z, (s0 + j) * SEG + 8 * lane, A.vocab, v[j]);
  const double c = octaves_per_logit(A, r);
  int rank[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    float top = v[j][0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = max_nan(top, v[j][e]);
    rank[j] = rank_of(top);
  }
  auto step = [&](auto ctrl) {
#pragma unroll
    for (int j = 0; j < U; ++j) rank[j] = max_moved<decltype(ctrl)::value>(rank[j]);
  };
  step(std::integral_constant<int, 0x111>{});
  step(std::integral_constant<int, 0x112>{});
  step(std::integral_constant<int, 0x114>{});
  if constexpr (CUT) {                            // lanes 7, 15, ..: of eight lanes
#pragma unroll
    for (int j = 0; j < U; ++j)
      if ((lane & 7) == 7 && s0 + j < segs) A.strip_m[((int64_t)r * segs + s0 + j) * 8 + (lane >> 3)] = of_rank(rank[j]);
  }
  step(std::integral_constant<int, 0x118>{});
  step(std::integral_constant<int, 0x142>{});
  step(std::integral_constant<int, 0x143>{});
  bool plain = true;                              // finite maxima, z c - m c good to 2^-44
  double mc[U], s[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    m[j] = of_rank(__builtin_amdgcn_readlane(rank[j], 63));
    mc[j] = (double)m[j] * c;
    plain = plain && fabs(mc[j]) < 1024.0;
    s[j] = 0.0;
  }
  const Exp2 exp2;
  if (plain) {
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[j] += exp2(fmax(fma((double)v[j][e], c, -mc[j]), -1000.0));
  } else {
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (m[j] > -INFINITY && m[j] < INFINITY)    // else the sum is not looked at, or nothing
#pragma unroll
        for (int e = 0; e < 8; ++e) s[j] += weight_of(v[j][e], m[j], c);
  }
#pragma unroll
  for (int j = 0; j < U; ++j) s[j] = sum_to_63(s[j]);
#pragma unroll
  for (int j = 0; j < U; ++j)
    if (lane == 63 && s0 + j < segs) {
      A.seg_m[(int64_t)r * segs + s0 + j] = m[j];
      A.seg_s[(int64_t)r * segs + s0 + j] = s[j];
    }
  if (CUT && A.bins) {                            // the histogram begins empty
    const int per = (BINS + (int)per_row - 1) / (int)per_row, b0 = s0 / U * per;
    for (int i = b0 + lane; i < min(b0 + per, BINS); i += 64) A.bins[(int64_t)r * BINS + i] = 0;
  }
}

// ---------------------------------------------------------------- a row
// Order of z as whole numbers, and back.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z == 0.f ? 0.f : z);       // -0 is 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
// A token's place in the order, its own: a larger one comes first.
__device__ __forceinline__ u64 place_of(float z, int id) {
  return (u64)key_of(z) << ID_BITS | (uint32_t)((1 << ID_BITS) - 1 - id);
}
__device__ __forceinline__ float z_of(u64 place) { return of_key((uint32_t)(place >> ID_BITS)); }
__device__ __forceinline__ int id_of(u64 place) { return (1 << ID_BITS) - 1 - (int)(place & ((1 << ID_BITS) - 1)); }

// Over a workgroup of N threads; `red` holds a value a wave.
template <int N, typename V>
__device__ __forceinline__ V group_prefix(V v, V* red, V* total) {   // inclusive
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const V y = __shfl_up(v, o, 64);
    if (lane >= o) v += y;
  }
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
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if (lane == 0) red[w] = v;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N / 64; ++i) v = min(v, red[i]);
  return v;
}
template <typename V>
__device__ __forceinline__ V wave_prefix(V v) {                      // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const V y = __shfl_up(v, o, 64);
    if (lane >= o) v += y;
  }
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

// Bin of z, 16 an octave of weight: falls as z grows.
__device__ __forceinline__ int bin_of(float z, float zmax, float c) {
  return (int)fminf(((zmax - z) * c) * 16.f, (float)(BINS - 1));
}
__device__ __forceinline__ float bin_factor(double c) { return (float)fmin(c, 3.0e38); }
// Weight, or u of it, at which top-p ends: the first token is always kept.
__device__ __forceinline__ double mass_limit(const RowOpts& o, double all) { return fmax((double)o.top_p * all, 0.5); }
// Which rows go by histogram: top-k's are few and the pick finds them alone.
__device__ __forceinline__ bool by_bins(const RowOpts& o) { return o.temperature != 0.0 && !o.by_k && (o.by_p || o.by_min); }
// min-p's border: the least fp32 value that is not below max z + T ln(min_p).
__device__ __forceinline__ float min_p_border(const RowOpts& o, float zmax) {
  const double lowest = (double)zmax + o.temperature * log(fmin(o.min_p, 1.0));
  const float t = (float)lowest;
  return (double)t < lowest ? of_key(key_of(t) + 1) : t;
}
// Part p of a row's segments: a run of them.
__device__ __forceinline__ int part_start(int p, int segs, int parts) { return (int)((int64_t)p * segs / parts); }

// The segments of a row, for one wave: lane l has those numbered l + 64 j, the first REGS
// in registers, others from memory again and again.
struct Segments {
  static constexpr int REGS = 8;      // 262144 tokens
  const float* top_of;
  const double* sum_of;
  int segs;
  float zmax;
  double c, total;
  float top[REGS];
  double share[REGS];

  __device__ __forceinline__ double share_of(float m, double s) const { return m == -INFINITY ? 0.0 : s * weight_of(m, zmax, c); }
  // f(index, maximum, share) for every segment of the lane, in order; past the last -inf and 0
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < REGS; ++j)
      if (64 * j < segs) f(lane + 64 * j, top[j], share[j]);
#pragma unroll 1
    for (int i = lane + 64 * REGS; i - lane < segs; i += 64) {
      const float m = i < segs ? top_of[i] : -INFINITY;
      f(i, m, i < segs ? share_of(m, sum_of[i]) : 0.0);
    }
  }
  // False where the row has no answer.
  __device__ __forceinline__ bool read(const DrawArgs& A, int r, int n, const RowOpts& o) {
    const int lane = threadIdx.x & 63;
    top_of = A.seg_m + (int64_t)r * n;
    sum_of = A.seg_s + (int64_t)r * n;
    segs = n;
    c = o.c;
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < REGS; ++j) {
      const int i = lane + 64 * j;
      top[j] = i < segs ? top_of[i] : -INFINITY;
      share[j] = i < segs ? sum_of[i] : 0.0;
    }
#pragma unroll
    for (int j = 0; j < REGS; ++j) m = max_nan(m, top[j]);
#pragma unroll 1
    for (int i = lane + 64 * REGS; i < segs; i += 64) m = max_nan(m, top_of[i]);
    zmax = max_nan_wave(m);
    if (!(zmax > -INFINITY && zmax < INFINITY) || !usable(o)) return false;   // NaN too
    double part = 0.0;
#pragma unroll
    for (int j = 0; j < REGS; ++j)
      if (64 * j < segs) {
        share[j] = share_of(top[j], share[j]);
        part += share[j];
      }
#pragma unroll 1
    for (int i = lane + 64 * REGS; i < segs; i += 64) part += share_of(top_of[i], sum_of[i]);
    total = from_63(sum_to_63(part));
    return true;
  }
  // The least z that can be kept (see above), the octaves that are left halved again and
  // again.  strips (n_strips of them, or none): taken in the place of the segments.
  __device__ __forceinline__ float least(const float* strips, int n_strips, int k, bool by_p, double p) const {
    const int lane = threadIdx.x & 63;
    float lo = 0.f, hi = FIXED_OCTAVES;
    if (by_p || (k > 0 && k <= max(n_strips, segs))) {
      const float spare = (float)((1.0 - fmax(p, 0.0)) * total * (1.0 - 1e-5)), cf = bin_factor(c);
#pragma unroll 1
      for (int round = 0; round < 8; ++round) {
        const float y = 0.5f * (lo + hi);
        bool pass;
        if (by_p) {
          const float cap = (float)SEG * __builtin_amdgcn_exp2f(-y);
          float below = 0.f;
          each([&](int, float m, double part) { below += (zmax - m) * cf <= y ? fminf((float)part, cap) : (float)part; });
          pass = sum_wave(below) <= spare;
        } else {
          int count = 0;
          if (n_strips) {
#pragma unroll 4
            for (int i = lane; i < n_strips; i += 64) count += (zmax - strips[i]) * cf <= y;
            count = wave_sum_dpp(count);
          } else {
            each([&](int, float m, double) { count += __popcll(__ballot((zmax - m) * cf <= y)); });
          }
          pass = count >= k;
        }
        if (pass) hi = y;
        else lo = y;
      }
    }
    const float t = (float)((double)zmax - ((double)hi + 2e-3) / c);
    return t <= -3.4e38f ? -INFINITY : of_key(key_of(t) - 2);   // 2e-3 and two steps: what was rounded on the way
  }
};

// Where f of a row's tokens can be had from: its logits.
template <typename T, bool VEC>
struct Logits {
  const T* z;
  int vocab;
  float zmax;
  double c;

  __device__ __forceinline__ u64 fixed(float x) const { return x == -INFINITY ? 0 : fixed_of(weight_of(x, zmax, c)); }
  // f(segment, its tokens' z, 8 a lane, the first's id) for the segments s0 .. s1 - 1 that
  // have a token of t0 or more, by their maxima top_of; called by N threads, whose waves
  // take them in turn, four on their way at once.
  template <int N, typename F>
  __device__ __forceinline__ void segments(uint16_t (&seg)[N / 64][MAX_SEGS * 64 / N + 1], const float* top_of, float t0, int s0,
                                           int s1, F f) const {
    constexpr int W = N / 64, U = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    int found = 0;
#pragma unroll 2
    for (int base = s0; base < s1; base += 64) {
      const float top = base + lane < s1 ? top_of[base + lane] : -INFINITY;
      const bool on = top >= t0 && top > -INFINITY;
      const uint64_t mask = __ballot(on);
      const int at = found + __popcll(mask & ((1ull << lane) - 1));
      if (on && at % W == wave) seg[wave][at / W] = (uint16_t)(base + lane);
      found += __popcll(mask);
    }
    const int n = (found - wave + W - 1) / W;
#pragma unroll 1
    for (int a = 0; a < n; a += U) {
      float v[U][8];
      int s[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        s[j] = a + j < n ? __builtin_amdgcn_readfirstlane((int)seg[wave][a + j]) : -1;
        load8<T, VEC>(z, s[j] < 0 ? vocab : s[j] * SEG + 8 * lane, vocab, v[j]);
      }
#pragma unroll
      for (int j = 0; j < U; ++j)
        if (s[j] >= 0) f(s[j], v[j], s[j] * SEG + 8 * lane);
    }
  }
  // f(z, id) for their tokens of t0 or more.
  template <int N, typename F>
  __device__ __forceinline__ void tokens(uint16_t (&seg)[N / 64][MAX_SEGS * 64 / N + 1], const float* top_of, float t0, int s0,
                                         int s1, F f) const {
    segments<N>(seg, top_of, t0, s0, s1, [&](int, const float (&v)[8], int first) {
      float top = v[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, v[e]);
      if (top >= t0 && top > -INFINITY)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (v[e] >= t0 && v[e] > -INFINITY) f(v[e], first + e);   // tokens past the vocabulary are -inf
    });
  }
  // By one wave: the token of segment s at which the running sum of weigh(z, id), `before` in
  // front of the segment, passes `want`; the last with a weight where none does.
  template <typename V, typename W>
  __device__ __forceinline__ int token_at(int s, V before, double want, W weigh, float& at) const {
    const int first = s * SEG + 8 * ((int)threadIdx.x & 63);
    float v[8];
    load8<T, VEC>(z, first, vocab, v);
    V w[8], sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = first + e < vocab ? weigh(v[e], first + e) : 0;
      sum += w[e];
    }
    V run = wave_prefix(sum) + before - sum;
    int hit = INT32_MAX, last = -1;
    float z_hit = 0.f, z_last = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      run += w[e];
      if (w[e] > 0) {
        last = first + e;
        z_last = v[e];
        if (hit == INT32_MAX && (double)run > want) {
          hit = first + e;
          z_hit = v[e];
        }
      }
    }
    const uint64_t hits = __ballot(hit != INT32_MAX), lasts = __ballot(last >= 0);
    const int from = hits ? first_lane(hits) : last_lane(lasts | 1);
    at = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(hits ? z_hit : z_last), from));
    return __builtin_amdgcn_readlane(hits ? hit : last, from);
  }
};

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

__device__ __forceinline__ double given_u(const DrawArgs& A, int r) {
  return A.u64 ? ((const double*)A.u)[r] : (double)((const float*)A.u)[r];
}
__device__ __forceinline__ void no_answer(const DrawArgs& A, int r) {
  A.token[r] = -1;
  A.logprob[r] = A.kept[r] = __uint_as_float(0x7FC00000u);
}
__device__ __forceinline__ void answer(const DrawArgs& A, int r, int id, float z, float zmax, double c, double total, double kept) {
  const double lw = ((double)z - (double)zmax) * c * 0.6931471805599453;
  A.token[r] = id;
  A.logprob[r] = (float)(lw - log(total));
  A.kept[r] = (float)(lw - log(kept));
}

// By one wave: a row of which nothing is cut, or all but the first of the largest (T = 0).
template <typename T, bool VEC>
__device__ __forceinline__ void draw_plain(const DrawArgs& A, int r, const Segments& S, const Logits<T, VEC>& z, const RowOpts& o,
                                           double u) {
  double want = u * S.total, before = 0.0;
  float at_z;
  int at = -1, id;
  if (o.temperature == 0.0) {
    S.each([&](int i, float m, double) {
      const uint64_t mask = __ballot(m == S.zmax);
      if (at < 0 && mask) at = __builtin_amdgcn_readfirstlane(i) + first_lane(mask);
    });
    id = z.token_at(at, 0.0, 0.0, [&](float x, int) { return x == S.zmax ? 1.0 : 0.0; }, at_z);
  } else {
    int last = 0;
    S.each([&](int i, float, double w) {
      if (at >= 0) return;
      const double end = wave_prefix(w) + before;
      const uint64_t past = __ballot(w > 0.0 && end > want), some = __ballot(w > 0.0);
      const int base = __builtin_amdgcn_readfirstlane(i);
      if (past) {
        at = base + first_lane(past);
        before = lane_of(end - w, first_lane(past));
      } else {
        if (some) last = base + last_lane(some);
        before = lane_of(end, 63);
      }
    });
    if (at < 0) {                     // roundings next to u = 1
      at = last;
      want = INFINITY;
    }
    id = z.token_at(at, before, want, [&](float x, int) { return x == -INFINITY ? 0.0 : weight_of(x, S.zmax, S.c); }, at_z);
  }
  if ((threadIdx.x & 63) == 0) {
    answer(A, r, id, at_z, S.zmax, S.c, S.total, S.total);
    if (o.temperature == 0.0) A.kept[r] = 0.f;
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_draw_plain(DrawArgs A, int segs) {
  const int r = (int)(blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6));
  if (r >= A.rows) return;
  const RowOpts o = row_opts(A, r);
  const double u = given_u(A, r);
  Segments S;
  if (!S.read(A, r, segs, o) || !(u >= 0.0 && u < 1.0)) {
    if ((threadIdx.x & 63) == 0) no_answer(A, r);
    return;
  }
  draw_plain<T, VEC>(A, r, S, Logits<T, VEC>{(const T*)A.logits + r * A.row, A.vocab, S.zmax, S.c}, o, u);
}

// ---------------------------------------------------------------- rows, bins, collect
__global__ __launch_bounds__(256) void k_draw_rows(DrawArgs A, int segs) {
  const int r = (int)(blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6));
  if (r >= A.rows) return;
  const RowOpts o = row_opts(A, r);
  if (!by_bins(o)) return;
  Segments S;
  const bool good = S.read(A, r, segs, o);
  float t0 = 0.f;
  if (good) {
    t0 = S.least(nullptr, 0, 0, o.by_p, o.top_p);
    if (o.by_min) t0 = fmaxf(t0, min_p_border(o, S.zmax));
  }
  if ((threadIdx.x & 63) == 0) A.info[r] = DrawRow{S.total, S.zmax, t0, good, 0, BINS, 0};
}

template <typename T, bool VEC>
__global__ __launch_bounds__(PART) void k_draw_bins(DrawArgs A, int segs, int parts) {
  __shared__ uint16_t active[PART / 64][MAX_SEGS * 64 / PART + 1];
  __shared__ u64 mass[BINS];
  const int r = blockIdx.x / parts, part = blockIdx.x - r * parts, tid = threadIdx.x;
  const RowOpts o = row_opts(A, r);
  if (!by_bins(o)) return;
  const DrawRow info = A.info[r];
  if (!info.good) return;
  for (int i = tid; i < BINS; i += PART) mass[i] = 0;
  __syncthreads();
  const float c = bin_factor(o.c);
  const Logits<T, VEC> z{(const T*)A.logits + r * A.row, A.vocab, info.zmax, o.c};
  z.template tokens<PART>(active, A.seg_m + (int64_t)r * segs, info.t0, part_start(part, segs, parts),
                          part_start(part + 1, segs, parts),
                          [&](float x, int) { atomicAdd(&mass[bin_of(x, info.zmax, c)], z.fixed(x)); });
  __syncthreads();
  u64* bins = A.part_bins + (int64_t)blockIdx.x * BINS;
  for (int i = tid; i < BINS; i += PART) {
    const u64 m = mass[i];
    bins[i] = m;
    if (m) atomicAdd(&A.bins[(int64_t)r * BINS + i], m);
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(PART) void k_draw_collect(DrawArgs A, int segs, int parts) {
  __shared__ uint16_t active[PART / 64][MAX_SEGS * 64 / PART + 1];
  __shared__ u64 red[8], list[LIST];
  __shared__ int redi[8], n_list, at;
  const int r = blockIdx.x / parts, part = blockIdx.x - r * parts, tid = threadIdx.x;
  const RowOpts o = row_opts(A, r);
  if (!by_bins(o)) return;
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
  int border = BINS;                  // the bin in which top-p's border lies
  if (o.by_p) {
    const double limit = mass_limit(o, info.total * FIXED_ONE);
    u64 sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += mine[i];
    u64 end = group_prefix<PART>(sum, red, &all);
    int hit = BINS;
    u64 before = end;
#pragma unroll
    for (int i = PER - 1; i >= 0; --i) {
      if (mine[i] && (double)end >= limit) {
        hit = tid * PER + i;
        before = end - mine[i];
      }
      end -= mine[i];
    }
    border = group_min<PART>(hit, redi);
    if (part == 0 && hit == border && border < BINS) {
      A.info[r].bin = border;
      A.info[r].above = before;
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (tid * PER + i < border) kept += own[i];       // what the part keeps above it
  group_prefix<PART>(kept, red, &all);
  if (tid == 0) A.part_kept[blockIdx.x] = all;
  if (border == BINS) return;
  const float c = bin_factor(o.c);
  const Logits<T, VEC> z{(const T*)A.logits + r * A.row, A.vocab, info.zmax, o.c};
  z.template tokens<PART>(active, A.seg_m + (int64_t)r * segs, info.t0, part_start(part, segs, parts),
                          part_start(part + 1, segs, parts), [&](float x, int id) {
                            if (bin_of(x, info.zmax, c) != border) return;
                            const int k = atomicAdd(&n_list, 1);
                            if (k < LIST) list[k] = place_of(x, id);
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
struct CutMemory {
  union {
    struct { u64 mass[BINS]; uint32_t count[BINS]; } bin;
    u64 seg[MAX_SEGS];                // kept weight of each segment
  };
  u64 list[LIST];                     // places of the tokens that can be kept
  uint16_t active[PICK / 64][MAX_SEGS * 64 / PICK + 1];
  u64 few[FEW], weight[FEW];
  u64 red[8], found, mass, rank, lo, hi;
  int redi[8], n_list, n_few;
};

// By one wave, a token (place p, weight w) in each of the first n lanes: how many of them
// come before the lane's, and what those weigh.
__device__ __forceinline__ void compare(int n, u64 p, u64 w, int& rank, u64& before) {
#pragma unroll 1
  for (int j = 0; j < n; ++j) {
    const bool in_front = lane_of(p, j) > p;
    rank += in_front;
    before += in_front ? lane_of(w, j) : 0;
  }
}

// The border of top-k (by rank: fewer than `limit` tokens come before) or top-p (less
// than `limit` of weight does) among the tokens that `each` gives, n of them, mass0 of
// weight in front of them, none outside the places lo .. hi: the place of the last that is
// kept, 0 if all of them are; mass: the weight up to it.  Windows of places, ever finer by
// 1024, until a wave can compare what is left.
template <typename R, typename Each>
__device__ __forceinline__ u64 find_border(const R& row, CutMemory& C, const Each& each, int n, bool by_rank, double limit, u64 lo,
                                           u64 hi, u64 mass0, u64* mass) {
  const int tid = threadIdx.x;
  constexpr int PER = BINS / PICK;
  u64 rank0 = 0;                      // before the window
  int inside = n;
  auto reaches = [&](u64 rank, u64 weight) { return by_rank ? (double)rank >= limit : (double)weight >= limit; };
#pragma unroll 1
  while (inside > FEW) {              // places differ: at the latest a window of one has one token
    __syncthreads();
    for (int i = tid; i < BINS; i += PICK) { C.bin.mass[i] = 0; C.bin.count[i] = 0; }
    __syncthreads();
    const int shift = max(54 - __clzll((long long)(hi - lo | 1)), 0);   // (hi - lo) >> shift is below 1024
    each([&](float x, int id) {
      const u64 p = place_of(x, id);
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
    m = group_prefix<PICK>(m, C.red, &all_m) + mass0;
    rank = group_prefix<PICK>(rank, C.red, &all_n) + rank0;
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
    const int d = group_min<PICK>(hit, C.redi);
    if (d == INT32_MAX) {             // the limit lies behind the last token
      *mass = mass0 + all_m;
      return 0;
    }
    if (hit == d) {
      C.mass = hit_m;
      C.rank = hit_n;
    }
    __syncthreads();
    mass0 = C.mass;
    rank0 = C.rank;
    inside = (int)min(C.bin.count[d], (uint32_t)FEW + 1);
    lo += (u64)(BINS - 1 - d) << shift;
    hi = min(hi, lo + ((1ull << shift) - 1));
  }
  __syncthreads();
  if (tid == 0) C.n_few = 0;
  __syncthreads();
  each([&](float x, int id) {
    const u64 p = place_of(x, id);
    if (p >= lo && p <= hi) {
      const int i = atomicAdd(&C.n_few, 1);
      C.few[i] = p;
      C.weight[i] = row.fixed(x);
    }
  });
  __syncthreads();
  if (tid < 64) {
    const int k = C.n_few;
    const u64 p = tid < k ? C.few[tid] : 0, w = tid < k ? C.weight[tid] : 0;
    int rank = 0;
    u64 before = mass0;
    compare(k, p, w, rank, before);
    const uint64_t ends = __ballot(tid < k && !reaches(rank0 + rank, before) && reaches(rank0 + rank + 1, before + w));
    const u64 all = lane_of(wave_prefix(w), 63);
    if (tid == 0) {
      C.found = ends ? 1 : 0;
      C.mass = mass0 + all;           // the limit lies behind the last token
    }
    if (ends && tid == first_lane(ends)) {
      C.found = p;
      C.mass = before + w;
    }
  }
  __syncthreads();
  *mass = C.mass;
  return C.found;
}

template <typename T, bool VEC>
__global__ __launch_bounds__(PICK) void k_draw_pick(DrawArgs A, int segs, int parts) {
  __shared__ CutMemory C;
  const int r = blockIdx.x, tid = threadIdx.x;
  const RowOpts o = row_opts(A, r);
  const double u = given_u(A, r);
  const bool binned = by_bins(o);
  DrawRow info{};
  Segments S;
  float t0 = 0.f;                     // no token below it is kept
  if (binned) {
    info = A.info[r];
    t0 = info.t0;
    S.segs = segs;
    S.top_of = A.seg_m + (int64_t)r * segs;
    S.zmax = info.zmax;
    S.total = info.total;
    S.c = o.c;
  } else {
    info.good = S.read(A, r, segs, o);   // every wave alike: none waits for another
  }
  if (!info.good || !(u >= 0.0 && u < 1.0)) {
    if (tid == 0) no_answer(A, r);
    return;
  }
  const Logits<T, VEC> z{(const T*)A.logits + r * A.row, A.vocab, S.zmax, S.c};
  if (!binned && (o.temperature == 0.0 || !o.by_k)) {   // nothing is cut here
    if (tid < 64) draw_plain<T, VEC>(A, r, S, z, o, u);
    return;
  }
  const float min_z = o.by_min ? min_p_border(o, S.zmax) : -INFINITY;
  u64 border = o.by_min ? (u64)key_of(min_z) << ID_BITS : 0;
  const bool whole_list = binned && info.listed <= LIST;   // the border's bin is listed, the rest summed
  if (!binned) {
    float* const strips = reinterpret_cast<float*>(C.list);   // where k is too many for the segments
    int n_strips = 0;
    if (2 * o.top_k > segs && 4 * segs <= LIST) {
      n_strips = 8 * segs;
      for (int i = tid; i < n_strips; i += PICK) strips[i] = A.strip_m[(int64_t)r * n_strips + i];
      __syncthreads();
    }
    t0 = S.least(strips, n_strips, o.top_k, false, 1.0);
    if (!o.by_p) t0 = fmaxf(t0, min_z);                    // top-p takes its share of all the k
    __syncthreads();
  }
  if (tid == 0) {
    C.n_list = whole_list ? info.listed : 0;
    C.lo = ~0ull;
    C.hi = 0;
  }
  __syncthreads();
  if (whole_list) {
    for (int i = tid; i < info.listed; i += PICK) C.list[i] = A.list[(int64_t)r * LIST + i];
  } else {
    z.template tokens<PICK>(C.active, S.top_of, t0, 0, segs, [&](float x, int id) {
      const int i = atomicAdd(&C.n_list, 1);
      if (i < LIST) C.list[i] = place_of(x, id);
    });
  }
  __syncthreads();
  const int n_list = C.n_list;

  // Few of all that can be kept: a lane each of one wave, compared with one another and
  // drawn from by their ids.
  if (!whole_list && n_list <= FEW) {
    if (tid >= 64) return;
    const bool is = tid < n_list;
    const u64 p = is ? C.list[tid] : 0, w = is ? z.fixed(z_of(p)) : 0;
    const int id = is ? id_of(p) : INT32_MAX;
    int rank = 0;
    u64 before = 0, all = 0;
    compare(n_list, p, w, rank, before);
    bool in = is && (!o.by_k || rank < o.top_k);
    if (o.by_p) {
      const double share = o.by_k ? (double)lane_of(wave_prefix(in ? w : 0), 63) : S.total * FIXED_ONE;
      in = in && (double)before < mass_limit(o, share);
    }
    in = in && p >= border;
    u64 end = 0;
#pragma unroll 1
    for (uint64_t left = __ballot(in); left; left &= left - 1) {
      const int j = first_lane(left);
      const u64 x = lane_of(w, j);
      all += x;
      end += __builtin_amdgcn_readlane(id, j) <= id ? x : 0;
    }
    const double want = u * (double)all;
    const uint64_t past = __ballot(in && w > 0 && (double)end > want), some = __ballot(in && w > 0);
    // the lowest id of those past it; roundings next to u = 1: the highest with a weight
    int hit = past ? INT32_MAX : -1;
#pragma unroll 1
    for (uint64_t left = past ? past : some; left; left &= left - 1) {
      const int x = __builtin_amdgcn_readlane(id, first_lane(left));
      hit = past ? min(hit, x) : max(hit, x);
    }
    if (in && id == hit) answer(A, r, id, z_of(p), S.zmax, S.c, S.total, (double)all / FIXED_ONE);
    return;
  }

  auto each = [&](auto f) {
    if (n_list <= LIST) {
      for (int i = tid; i < n_list; i += PICK) f(z_of(C.list[i]), id_of(C.list[i]));
    } else {
      z.template tokens<PICK>(C.active, S.top_of, t0, 0, segs, f);
    }
  };
  u64 lo = place_of(t0, (1 << ID_BITS) - 1), hi = place_of(S.zmax, 0);
  if (n_list <= LIST) {               // no wider than the list is
    u64 least = ~0ull, most = 0;
    for (int i = tid; i < n_list; i += PICK) {
      least = min(least, C.list[i]);
      most = max(most, C.list[i]);
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) {
      least = min(least, __shfl_xor(least, x, 64));
      most = max(most, __shfl_xor(most, x, 64));
    }
    if ((tid & 63) == 0) {
      atomicMin(&C.lo, least);
      atomicMax(&C.hi, most);
    }
    __syncthreads();
    lo = C.lo;
    hi = C.hi;
  }
  double share = S.total * FIXED_ONE;
#pragma unroll 1
  for (int rule = 0; rule < 2; ++rule) {
    if (rule == 0 ? !o.by_k : !o.by_p || (whole_list && info.bin == BINS)) continue;
    u64 mass;
    border = max(border, find_border(z, C, each, n_list, rule == 0, rule == 0 ? (double)o.top_k : mass_limit(o, share), lo, hi,
                                     whole_list ? info.above : 0, &mass));
    share = (double)mass;
  }
  // What is kept of each segment or, where the histogram knows the parts', of each part
  // and then of that part's segments.
  __syncthreads();
  const int lane = tid & 63;
  int s0 = 0, s1 = segs;
  u64 before = 0, kept = 0;
  double want = 0.0;
  if (whole_list) {
    for (int i = tid; i < parts; i += PICK) C.seg[i] = A.part_kept[(int64_t)r * parts + i];
    __syncthreads();
    for (int i = tid; i < n_list; i += PICK)
      if (C.list[i] >= border) {
        const int s = id_of(C.list[i]) / SEG;
        int p = (int)((int64_t)s * parts / segs);
        while (part_start(p + 1, segs, parts) <= s) ++p;
        atomicAdd(&C.seg[p], z.fixed(z_of(C.list[i])));
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
  for (int i = tid; i < segs; i += PICK) C.seg[i] = 0;
  __syncthreads();
  if (!whole_list && n_list <= LIST) {
    each([&](float x, int id) {
      if (place_of(x, id) >= border) atomicAdd(&C.seg[id / SEG], z.fixed(x));
    });
  } else {                            // a segment's tokens add up within their wave
    z.template segments<PICK>(C.active, S.top_of, t0, s0, s1, [&](int s, const float (&v)[8], int first) {
      u64 sum = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (v[e] >= t0 && place_of(v[e], first + e) >= border) sum += z.fixed(v[e]);
#pragma unroll
      for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x, 64);
      if (lane == 0) C.seg[s] = sum;
    });
  }
  __syncthreads();
  if (tid >= 64) return;
  if (!whole_list) {
    for (int i = lane; i < segs; i += 64) kept += C.seg[i];
    kept = lane_of(wave_prefix(kept), 63);
    want = u * (double)kept;
  }
  const int at = s0 + entry_at(s1 - s0, [&](int i) { return C.seg[s0 + i]; }, want, before);
  float at_z;
  const int id = z.token_at(at, before, want, [&](float x, int i) { return place_of(x, i) >= border ? z.fixed(x) : (u64)0; }, at_z);
  if (lane == 0) answer(A, r, id, at_z, S.zmax, S.c, S.total, (double)kept / FIXED_ONE);
}

int segments(int vocab) { return (vocab + SEG - 1) / SEG; }

// Whether rows may be cut, and whether some may go by histogram.
bool may_cut(const DrawArgs& a) { return a.top_k_rows || a.top_p_rows || a.min_p_rows || a.top_k > 0 || a.top_p < 1.0 || a.min_p > 0.0; }
bool may_bin(const DrawArgs& a) {
  return (a.top_k_rows || a.top_k == 0 || a.top_k >= a.vocab) && (a.top_p_rows || a.min_p_rows || a.top_p < 1.0 || a.min_p > 0.0);
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
  s.end = (s.strip_m + (may_cut(a) ? 32 * n : 0) + 15) / 16 * 16;
  return s;
}

template <typename T, bool VEC>
hipError_t run(const DrawArgs& a, hipStream_t st) {
  const int segs = segments(a.vocab);
  const unsigned per_row = (unsigned)(segs + 3) / 4;
  const int64_t items = (int64_t)a.rows * per_row;
  if (items > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((items + SCAN_WAVES - 1) / SCAN_WAVES)), scan(64 * SCAN_WAVES), row(PICK);
  hipError_t e;
  const dim3 waves((unsigned)((a.rows + 3) / 4)), four(256);
  if (!may_cut(a)) {
    if ((e = kv8_launch(k_draw_scan<T, VEC, false>, grid, scan, st, a, segs, per_row, (unsigned)items)) != hipSuccess) return e;
    return kv8_launch(k_draw_plain<T, VEC>, waves, four, st, a, segs);
  }
  if ((e = kv8_launch(k_draw_scan<T, VEC, true>, grid, scan, st, a, segs, per_row, (unsigned)items)) != hipSuccess) return e;
  const int parts = parts_of(a);
  if (a.bins) {
    if ((int64_t)a.rows * parts > INT32_MAX) return hipErrorInvalidValue;
    const dim3 g((unsigned)(a.rows * parts));
    if ((e = kv8_launch(k_draw_rows, waves, four, st, a, segs)) != hipSuccess) return e;
    if ((e = kv8_launch(k_draw_bins<T, VEC>, g, dim3(PART), st, a, segs, parts)) != hipSuccess) return e;
    if ((e = kv8_launch(k_draw_collect<T, VEC>, g, dim3(PART), st, a, segs, parts)) != hipSuccess) return e;
  }
  return kv8_launch(k_draw_pick<T, VEC>, dim3(a.rows), row, st, a, segs, parts);
}

}  // namespace

int64_t draw_scratch_bytes(const DrawArgs& a) { return scratch_of(a).end; }

hipError_t launch_draw(DrawArgs a, void* scratch, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  if (a.vocab < 1 || a.vocab > DRAW_MAX_VOCAB) return hipErrorInvalidValue;
  const Scratch s = scratch_of(a);
  char* p = (char*)scratch;
  a.c = a.temperature == 0.0 ? LOG2E : LOG2E / a.temperature;
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
