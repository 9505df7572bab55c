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
// * scan, a wave a segment of 512 tokens: maximum, and sum of weights with respect to
//   it.  It streams the logits once.
// * only where top-p or min-p may cut a row without top-k: histogram and collect, some
//   workgroups a row.  The first adds up weights by bins of z; the second finds the bin
//   in which the border of top-p lies, sums what is kept above it by segments, and
//   lists the tokens in it.
// * pick, a workgroup a row: the border, then the segment, then the token.
// The last three look only at segments that can hold kept tokens:
// * weights below 2^-43 of the largest count nothing;
// * k segments with a maximum of t or more hold k tokens of t or more, so the border of
//   top-k lies there or above;
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
constexpr int PICK = 512;             // threads of a row's pick
constexpr int PART = 256;             // threads of a part of a row's histogram
constexpr int BINS = 2 * PICK;        // of z, 16 an octave of weight
constexpr int LIST = 4096;            // tokens that a row's list holds
constexpr int FEW = 128;              // tokens that are put in order by comparing all of them
constexpr int ID_BITS = 20;
constexpr double LOG2E = 1.4426950408889634;
constexpr double FIXED_ONE = 4398046511104.0;   // 2^42
constexpr float FIXED_OCTAVES = 43.5f;          // weights below 2^-43 are 0 in whole numbers

// Settings of a row.
struct RowOpts {
  double temperature, top_p, min_p;
  int top_k;
  bool by_k, by_p, by_min;
  double c;                           // octaves of weight per logit; T = 0 reports at 1
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
  o.c = o.temperature == 0.0 ? LOG2E : LOG2E / o.temperature;
  return o;
}
__device__ __forceinline__ bool usable(const RowOpts& o) {
  return o.temperature >= 0.0 && o.temperature < (double)INFINITY && o.top_p == o.top_p && o.min_p == o.min_p;
}

// 2^t for t in [-1000, 1000]: 2^n times a polynomial of degree 8 that interpolates 2^f
// at the Chebyshev points of [-1/2, 1/2], 1.1e-12 relative.
__device__ __forceinline__ double exp2_64(double t) {
  constexpr double shifter = 6755399441055744.0;              // 1.5 * 2^52: the sum's low bits are t to nearest
  const double s = t + shifter, f = t - (s - shifter);
  double p = 1.3255224884799127e-06;
  p = fma(p, f, 1.5310079402383103e-05);
  p = fma(p, f, 0.00015403455852419016);
  p = fma(p, f, 0.0013333450568000008);
  p = fma(p, f, 0.00961812915940262);
  p = fma(p, f, 0.05550410941205934);
  p = fma(p, f, 0.2402265069581299);
  p = fma(p, f, 0.6931471805459335);
  p = fma(p, f, 1.0);
  const u64 b = __builtin_bit_cast(u64, p);
  return __builtin_bit_cast(double, b + ((u64)(uint32_t)__builtin_bit_cast(u64, s) << 52));
}
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

template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v) {            // lanes without a source: 0
  const u64 b = __builtin_bit_cast(u64, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (u64)hi << 32 | lo);
}
// Over the wave's lanes; the result is in lane 63.
__device__ __forceinline__ double sum_to_63(double v) {
  v += moved<0x111, 0xf>(v);          // row_shr 1, 2, 4, 8, then row_bcast 15 and 31
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);
  v += moved<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ float max_nan_wave(float v) {
#define RG_MAX(ctrl) \
  v = max_nan(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), ctrl, 0xf, 0xf, false)))
  RG_MAX(0x111);
  RG_MAX(0x112);
  RG_MAX(0x114);
  RG_MAX(0x118);
  RG_MAX(0x142);
  RG_MAX(0x143);
#undef RG_MAX
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

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
template <typename T, bool VEC>
__global__ __launch_bounds__(64 * SCAN_WAVES) void k_draw_scan(DrawArgs A, int segs, int64_t items) {
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * SCAN_WAVES + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (item >= items) return;
  const int r = (int)(item / segs), seg = (int)(item - (int64_t)r * segs);
  const double temperature = A.temperature_rows ? (double)A.temperature_rows[r] : A.temperature;
  const double c = temperature == 0.0 ? LOG2E : LOG2E / temperature;
  float v[8];
  load8<T, VEC>((const T*)A.logits + r * A.row, seg * SEG + 8 * lane, A.vocab, v);
  float m = v[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) m = max_nan(m, v[e]);
  m = max_nan_wave(m);
  double s = 0.0;
  if (m > -INFINITY && m < INFINITY) {            // else the sum is not looked at, or nothing
#pragma unroll
    for (int e = 0; e < 8; ++e) s += weight_of(v[e], m, c);   // the maximum's is 1 exactly
    s = sum_to_63(s);
  }
  if (lane == 63) {
    A.seg_m[item] = m;
    A.seg_s[item] = s;
  }
  if (A.bins) {                                   // the histogram begins empty
    const int per = (BINS + segs - 1) / segs;
    for (int i = seg * per + lane; i < min(seg * per + per, BINS); i += 64) A.bins[(int64_t)r * BINS + i] = 0;
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

// What the threads of a row share.
struct RowMemory {
  float m[MAX_SEGS];                  // maxima of the segments
  float share[MAX_SEGS];              // their sums with respect to the row's maximum
  uint16_t active[MAX_SEGS];          // segments that can hold kept tokens
  double redd[8];
  u64 red[8];
  float redf[8];
  int redi[8];
  int passes[8];
  int n_active;
};

template <typename T, bool VEC, int N>
struct Row {
  const T* z;
  int vocab, segs;
  float zmax;
  double c, total;
  RowMemory* S;

  // The row's segments; false where it has no answer.
  __device__ bool read(const DrawArgs& A, int r, int n_segs, const RowOpts& o) {
    const int tid = threadIdx.x;
    z = (const T*)A.logits + r * A.row;
    vocab = A.vocab;
    segs = n_segs;
    c = o.c;
    float m = -INFINITY;
    for (int i = tid; i < segs; i += N) {
      const float x = A.seg_m[(int64_t)r * segs + i];
      S->m[i] = x;
      m = max_nan(m, x);
    }
    m = max_nan_wave(m);
    if ((tid & 63) == 0) S->redf[tid >> 6] = m;
    __syncthreads();
    m = S->redf[0];
#pragma unroll
    for (int i = 1; i < N / 64; ++i) m = max_nan(m, S->redf[i]);
    zmax = m;
    if (!(zmax > -INFINITY && zmax < INFINITY) || !usable(o)) return false;   // NaN too
    double part = 0.0;
    for (int i = tid; i < segs; i += N) {
      const double w = share_of(A, r, i);
      S->share[i] = (float)w;
      part += w;
    }
    part = sum_to_63(part);
    if ((tid & 63) == 63) S->redd[tid >> 6] = part;
    __syncthreads();
    total = 0.0;
#pragma unroll
    for (int i = 0; i < N / 64; ++i) total += S->redd[i];
    return true;
  }
  __device__ double share_of(const DrawArgs& A, int r, int i) const {
    const float m = S->m[i];
    return m == -INFINITY ? 0.0 : A.seg_s[(int64_t)r * segs + i] * weight_of(m, zmax, c);
  }
  __device__ u64 fixed(float x) const { return x == -INFINITY ? 0 : fixed_of(weight_of(x, zmax, c)); }
  __device__ float octaves(float x) const { return (float)(((double)zmax - (double)x) * c); }

  // The least z that can be kept (see above), of min-p's z where given: thresholds side
  // by side, a wave each.
  __device__ float least(bool by_k, int k, bool by_p, double p, float min_z) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int W = N / 64;
    float lo = 0.f, hi = FIXED_OCTAVES;
    if (by_k || by_p) {
      const float spare = (float)((1.0 - fmax(p, 0.0)) * total * (1.0 - 1e-5));
      for (int round = 0; round < (W == 8 ? 3 : 4); ++round) {
        const float step = (hi - lo) / (W + 1), y = lo + step * (wave + 1);
        const float cap = (float)SEG * __builtin_amdgcn_exp2f(-y);
        float below = 0.f;
        int n = 0;
        for (int i = lane; i < segs; i += 64) {
          const bool above = octaves(S->m[i]) <= y;
          n += above;
          below += above ? fminf(S->share[i], cap) : S->share[i];
        }
        const bool pass = by_k ? wave_sum_dpp(n) >= k : wave_sum(below) <= spare;
        __syncthreads();
        if (lane == 0) S->passes[wave] = pass;
        __syncthreads();
        int first = W;
        for (int i = W - 1; i >= 0; --i)
          if (S->passes[i]) first = i;
        hi = first == W ? hi : lo + step * (first + 1);
        lo = lo + step * first;
      }
    }
    const float t = (float)((double)zmax - ((double)hi + 1e-3) / c);
    return fmaxf(t <= -3.4e38f ? -INFINITY : of_key(key_of(t) - 2), min_z);   // what was rounded on the way
  }
  // Lists the segments that can hold a token of t0 or more.
  __device__ void activate(float t0) {
    __syncthreads();
    if (threadIdx.x == 0) S->n_active = 0;
    __syncthreads();
    for (int base = 0; base < segs; base += N) {
      const int i = base + (int)threadIdx.x;
      const bool on = i < segs && S->m[i] >= t0;
      const uint64_t mask = __ballot(on);
      int at = 0;
      if ((threadIdx.x & 63) == 0 && mask) at = atomicAdd(&S->n_active, __popcll(mask));
      at = __builtin_amdgcn_readfirstlane(at);
      if (on) S->active[at + __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1))] = (uint16_t)i;
    }
    __syncthreads();
  }
  // f(z, id, whether it is a token of t0 or more) for the tokens of active segments; whole
  // waves call it.  Four segments are on their way at once.
  template <typename F>
  __device__ void from_memory(float t0, F f) const {
    constexpr int W = N / 64, U = 4;
    const int lane = threadIdx.x & 63, n = S->n_active;
    for (int a = (int)threadIdx.x >> 6; a < n; a += W * U) {
      float v[U][8];
      int first[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        first[j] = a + j * W < n ? (int)S->active[a + j * W] * SEG + 8 * lane : vocab;
        load8<T, VEC>(z, first[j], vocab, v[j]);
      }
#pragma unroll
      for (int j = 0; j < U; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) f(v[j][e], first[j] + e, first[j] + e < vocab && v[j][e] >= t0);
    }
  }
};

// min-p's border: the least fp32 value that is not below max z + T ln(min_p).
__device__ __forceinline__ float min_p_border(const RowOpts& o, float zmax) {
  const double lowest = (double)zmax + o.temperature * log(fmin(o.min_p, 1.0));
  const float t = (float)lowest;
  return (double)t < lowest ? of_key(key_of(t) + 1) : t;
}

// Which rows go by histogram: top-k's are few and the pick finds them alone.
__device__ __forceinline__ bool by_bins(const RowOpts& o) { return o.temperature != 0.0 && !o.by_k && (o.by_p || o.by_min); }

// Bin of z, 16 an octave of weight: falls as z grows.
__device__ __forceinline__ int bin_of(float z, float zmax, float c) {
  return (int)fminf(((zmax - z) * c) * 16.f, (float)(BINS - 1));
}
__device__ __forceinline__ float bin_factor(double c) { return (float)fmin(c, 3.0e38); }
__device__ __forceinline__ double mass_limit(const RowOpts& o, double all) { return fmax(o.top_p * all, 0.5); }

// Adds a token to a list where `on`; whole waves call it.
__device__ __forceinline__ void append(bool on, u64 place, int* count, u64* list) {
  const uint64_t mask = __ballot(on);
  if (!mask) return;
  const int lane = threadIdx.x & 63;
  int at = 0;
  if (lane == 0) at = atomicAdd(count, __popcll(mask));
  at = __builtin_amdgcn_readfirstlane(at) + __popcll(mask & ((1ull << lane) - 1));
  if (on && at < LIST) list[at] = place;
}

// ---------------------------------------------------------------- histogram, collect
template <typename T, bool VEC>
__global__ __launch_bounds__(PART) void k_draw_bins(DrawArgs A, int segs, int parts) {
  __shared__ RowMemory S;
  __shared__ u64 mass[BINS];
  const int r = blockIdx.x / parts, part = blockIdx.x - r * parts, tid = threadIdx.x;
  const RowOpts o = row_opts(A, r);
  if (!by_bins(o)) return;
  Row<T, VEC, PART> row{};
  row.S = &S;
  const bool good = row.read(A, r, segs, o);
  float t0 = 0.f;
  if (good) t0 = row.least(false, 0, o.by_p, o.top_p, o.by_min ? min_p_border(o, row.zmax) : -INFINITY);
  if (part == 0 && tid == 0) A.info[r] = DrawRow{row.total, row.zmax, t0, good, 0, BINS, 0};
  if (!good || !o.by_p) return;
  for (int i = tid; i < BINS; i += PART) mass[i] = 0;
  __syncthreads();
  const float c = bin_factor(o.c);
  const int lane = tid & 63;
  for (int s = part + parts * (tid >> 6); s < segs; s += parts * (PART / 64)) {
    if (S.m[s] < t0) continue;
    float v[8];
    load8<T, VEC>(row.z, s * SEG + 8 * lane, A.vocab, v);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (v[e] >= t0 && v[e] > -INFINITY) atomicAdd(&mass[bin_of(v[e], row.zmax, c)], row.fixed(v[e]));
  }
  __syncthreads();
  for (int i = tid; i < BINS; i += PART)
    if (mass[i]) atomicAdd(&A.bins[(int64_t)r * BINS + i], mass[i]);
}

template <typename T, bool VEC>
__global__ __launch_bounds__(PART) void k_draw_collect(DrawArgs A, int segs, int parts) {
  __shared__ u64 red[8];
  __shared__ int redi[8];
  const int r = blockIdx.x / parts, part = blockIdx.x - r * parts, tid = threadIdx.x;
  const RowOpts o = row_opts(A, r);
  if (!by_bins(o)) return;
  const DrawRow info = A.info[r];
  if (!info.good) return;
  int border = BINS;                  // the bin in which top-p's border lies
  u64 above = 0;                      // weight of the bins before it
  if (o.by_p) {
    const double limit = mass_limit(o, info.total * FIXED_ONE);
    constexpr int PER = BINS / PART;
    u64 mine[PER], sum = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      mine[i] = A.bins[(int64_t)r * BINS + tid * PER + i];
      sum += mine[i];
    }
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
    if (hit == border && border < BINS) red[0] = before;
    __syncthreads();
    above = border < BINS ? red[0] : 0;
  }
  if (part == 0 && tid == 0) {
    A.info[r].bin = border;
    A.info[r].above = above;
  }
  const T* z = (const T*)A.logits + r * A.row;
  const float c = bin_factor(o.c);
  const int lane = tid & 63;
  for (int s = part + parts * (tid >> 6); s < segs; s += parts * (PART / 64)) {
    u64 kept = 0;
    if (A.seg_m[(int64_t)r * segs + s] >= info.t0) {
      float v[8];
      const int i = s * SEG + 8 * lane;
      load8<T, VEC>(z, i, A.vocab, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool on = v[e] >= info.t0 && v[e] > -INFINITY;
        const int b = on ? bin_of(v[e], info.zmax, c) : BINS;
        if (b < border) kept += fixed_of(weight_of(v[e], info.zmax, o.c));
        append(b == border && on, place_of(v[e], i + e), &A.info[r].listed, A.list + (int64_t)r * LIST);
      }
#pragma unroll
      for (int x = 32; x > 0; x >>= 1) kept += __shfl_xor(kept, x, 64);
    }
    if (lane == 0) A.kept_seg[(int64_t)r * segs + s] = kept;
  }
}

// ---------------------------------------------------------------- pick
struct CutMemory {
  union {
    struct { u64 mass[BINS]; uint32_t count[BINS]; } bin;
    u64 seg[MAX_SEGS];                // kept weight of each segment
  };
  u64 list[LIST];                     // places of the tokens that can be kept
  u64 few[FEW], weight[FEW];
  u64 found, mass, rank;
  int n_list, n_few;
};

// The border of top-k (by rank: fewer than `limit` tokens come before) or top-p (less
// than `limit` of weight does) among the tokens that `each` gives, mass0 of weight in
// front of them, none outside the places lo .. hi: the place of the last that is kept, 0
// if all of them are; mass: the weight up to it.  Windows of places, ever finer by 1024,
// until what is left is few enough to compare with one another.
template <typename R, typename Each>
__device__ u64 find_border(const R& row, CutMemory& C, const Each& each, bool by_rank, double limit, u64 lo, u64 hi,
                           u64 mass0, u64* mass) {
  const int tid = threadIdx.x;
  u64 rank0 = 0;                      // before the window
  auto reaches = [&](u64 rank, u64 weight) { return by_rank ? (double)rank >= limit : (double)weight >= limit; };
  for (;;) {
    __syncthreads();
    for (int i = tid; i < BINS; i += PICK) { C.bin.mass[i] = 0; C.bin.count[i] = 0; }
    if (tid == 0) C.n_few = 0;
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
    const u64 m0 = C.bin.mass[2 * tid], m1 = C.bin.mass[2 * tid + 1];
    const uint32_t n0 = C.bin.count[2 * tid], n1 = C.bin.count[2 * tid + 1];
    u64 all_m, all_n;
    const u64 m = group_prefix<PICK>(m0 + m1, row.S->red, &all_m) + mass0;
    const u64 n = group_prefix<PICK>((u64)(n0 + n1), row.S->red, &all_n) + rank0;
    int hit = INT32_MAX;
    if (n1 && reaches(n, m)) hit = 2 * tid + 1;
    if (n0 && reaches(n - n1, m - m1)) hit = 2 * tid;
    const int d = group_min<PICK>(hit, row.S->redi);
    if (d == INT32_MAX) {             // the limit lies behind the last token
      *mass = mass0 + all_m;
      return 0;
    }
    if (hit == d) {
      C.mass = hit & 1 ? m - m1 : m - m1 - m0;
      C.rank = hit & 1 ? n - n1 : n - n1 - n0;
    }
    __syncthreads();
    mass0 = C.mass;
    rank0 = C.rank;
    const int inside = (int)min(C.bin.count[d], (uint32_t)FEW + 1);
    lo += (u64)(BINS - 1 - d) << shift;
    hi = min(hi, lo + ((1ull << shift) - 1));
    if (inside > FEW) continue;       // places differ: at the latest a window of one has one token
    each([&](float x, int id) {
      const u64 p = place_of(x, id);
      if (p >= lo && p <= hi) {
        const int i = atomicAdd(&C.n_few, 1);
        C.few[i] = p;
        C.weight[i] = row.fixed(x);
      }
    });
    __syncthreads();
    if (tid < inside) {
      const u64 p = C.few[tid];
      u64 before = mass0, rank = rank0;
      for (int j = 0; j < inside; ++j) {
        const bool in_front = C.few[j] > p;
        rank += in_front;
        before += in_front ? C.weight[j] : 0;
      }
      if (!reaches(rank, before) && reaches(rank + 1, before + C.weight[tid])) {
        C.found = p;
        C.mass = before + C.weight[tid];
      }
    }
    __syncthreads();
    *mass = C.mass;
    return C.found;
  }
}

template <typename T, bool VEC, bool CUT>
__global__ __launch_bounds__(PICK) void k_draw_pick(DrawArgs A, int segs) {
  __shared__ RowMemory S;
  __shared__ typename std::conditional<CUT, CutMemory, int>::type cut;
  __shared__ u64 start;
  const int r = blockIdx.x, tid = threadIdx.x;
  const RowOpts o = row_opts(A, r);
  const double u = A.u64 ? ((const double*)A.u)[r] : (double)((const float*)A.u)[r];
  Row<T, VEC, PICK> row{};
  row.S = &S;
  if (!row.read(A, r, segs, o) || !(u >= 0.0 && u < 1.0)) {
    if (tid == 0) {
      A.token[r] = -1;
      A.logprob[r] = A.kept[r] = __uint_as_float(0x7FC00000u);
    }
    return;
  }
  const double inv_t = o.temperature == 0.0 ? 1.0 : 1.0 / o.temperature;
  auto answer = [&](int id, float zi, double kept) {
    const double lw = ((double)zi - (double)row.zmax) * inv_t;
    A.token[r] = id;
    A.logprob[r] = (float)(lw - log(row.total));
    A.kept[r] = (float)(o.temperature == 0.0 ? 0.0 : lw - log(kept));
  };
  static_assert(PICK == SEG, "a thread a token of a segment");
  auto token = [&](int s) {
    const int i = s * SEG + tid;
    return i < A.vocab ? ld_f32<T>(row.z + i) : -INFINITY;
  };
  // The token of segment s at which the running sum, `before` in front of the segment,
  // passes `want`; w is the weight of the thread's token.
  auto finish = [&](int s, float zi, auto w, auto before, double want, double kept) {
    decltype(w) all;
    const auto end = group_prefix<PICK>(w, reinterpret_cast<decltype(w)*>(S.red), &all) + before;
    int hit = group_min<PICK>(w > 0 && (double)end > want ? tid : INT32_MAX, S.redi);
    if (hit == INT32_MAX) hit = -group_min<PICK>(w > 0 ? -tid : 1, S.redi);   // roundings next to u = 1: the last with a weight
    if (tid == hit) answer(s * SEG + tid, zi, kept);
  };
  // The first segment at whose end the running sum of f(segment) passes `want`, and the
  // sum in front of it.  Where roundings next to u = 1 leave none: the last that has a
  // weight, and nothing that its tokens could pass.
  auto find_segment = [&](auto f, double& want, auto& before) {
    using V = typename std::remove_reference<decltype(before)>::type;
    V run = 0;
    int last = 0;
    for (int base = 0; base < segs; base += PICK) {
      const int i = base + tid;
      const V w = i < segs ? f(i) : 0;
      V all;
      const V end = group_prefix<PICK>(w, reinterpret_cast<V*>(S.red), &all) + run;
      const int at = group_min<PICK>(w > 0 && (double)end > want ? i : INT32_MAX, S.redi);
      if (at != INT32_MAX) {
        if (i == at) *reinterpret_cast<V*>(&start) = end - w;
        __syncthreads();
        before = *reinterpret_cast<V*>(&start);
        return at;
      }
      last = max(last, -group_min<PICK>(w > 0 ? -i : 0, S.redi));
      run += all;
    }
    before = 0;
    want = INFINITY;
    return last;
  };

  if (o.temperature == 0.0) {         // the first of the largest
    int top = INT32_MAX;
    for (int i = tid; i < segs; i += PICK)
      if (S.m[i] == row.zmax) top = min(top, i);
    top = group_min<PICK>(top, S.redi);
    const float zi = token(top);
    const int at = group_min<PICK>(zi == row.zmax ? tid : INT32_MAX, S.redi);
    if (tid == at) answer(top * SEG + tid, zi, 1.0);
    return;
  }
  if (!CUT || !(o.by_k || o.by_p || o.by_min)) {   // every token can be drawn
    double before, want = u * row.total;
    const int at = find_segment([&](int i) { return row.share_of(A, r, i); }, want, before);
    const float zi = token(at);
    finish(at, zi, zi == -INFINITY ? 0.0 : weight_of(zi, row.zmax, row.c), before, want, row.total);
    return;
  }
  if constexpr (CUT) {
    CutMemory* const C = &cut;
    u64 border = 0, kept = 0;
    float t0;                         // no token below it is kept
    const float min_z = o.by_min ? min_p_border(o, row.zmax) : -INFINITY;
    if (o.by_min) border = (u64)key_of(min_z) << ID_BITS;
    DrawRow info{};
    bool binned = by_bins(o);
    if (binned) {
      info = A.info[r];
      binned = info.listed <= LIST;
      t0 = info.t0;
    } else {                          // top-p takes its share of all the k
      t0 = row.least(o.by_k, o.top_k, false, 1.0, o.by_p ? -INFINITY : min_z);
    }
    if (tid == 0) C->n_list = 0;
    row.activate(t0);
    int n_list;
    if (binned) {
      n_list = info.listed;
      for (int i = tid; i < n_list; i += PICK) C->list[i] = A.list[(int64_t)r * LIST + i];
    } else {
      row.from_memory(t0, [&](float x, int id, bool on) { append(on && x > -INFINITY, place_of(x, id), &C->n_list, C->list); });
      __syncthreads();
      n_list = C->n_list;
    }
    __syncthreads();
    auto each = [&](auto f) {
      if (n_list <= LIST) {
        for (int i = tid; i < n_list; i += PICK) f(z_of(C->list[i]), id_of(C->list[i]));
      } else {
        row.from_memory(t0, [&](float x, int id, bool on) {
          if (on && x > -INFINITY) f(x, id);
        });
      }
    };
    const u64 lo = place_of(t0, (1 << ID_BITS) - 1), hi = place_of(row.zmax, 0);
    if (o.by_k) {
      u64 mass;
      border = max(border, find_border(row, *C, each, true, (double)o.top_k, lo, hi, 0, &mass));
      if (o.by_p) border = max(border, find_border(row, *C, each, false, mass_limit(o, (double)mass), lo, hi, 0, &mass));
    } else if (o.by_p && !(binned && info.bin == BINS)) {
      u64 mass;
      border = max(border, find_border(row, *C, each, false, mass_limit(o, row.total * FIXED_ONE), lo, hi,
                                       binned ? info.above : 0, &mass));
    }
    __syncthreads();
    for (int i = tid; i < segs; i += PICK) C->seg[i] = binned ? A.kept_seg[(int64_t)r * segs + i] : 0;
    __syncthreads();
    each([&](float x, int id) {
      if (place_of(x, id) >= border) atomicAdd(&C->seg[id / SEG], row.fixed(x));
    });
    __syncthreads();
    u64 mine = 0, before;
    for (int i = tid; i < segs; i += PICK) mine += C->seg[i];
    group_prefix<PICK>(mine, S.red, &kept);
    double want = u * (double)kept;
    const int at = find_segment([&](int i) { return C->seg[i]; }, want, before);
    const float zi = token(at);
    const int id = at * SEG + tid;
    finish(at, zi, id < A.vocab && place_of(zi, id) >= border ? row.fixed(zi) : (u64)0, before, want, (double)kept / FIXED_ONE);
  }
}

int segments(int vocab) { return (vocab + SEG - 1) / SEG; }

// Whether rows may be cut, and whether some may go by histogram.
bool may_cut(const DrawArgs& a) { return a.top_k_rows || a.top_p_rows || a.min_p_rows || a.top_k > 0 || a.top_p < 1.0 || a.min_p > 0.0; }
bool may_bin(const DrawArgs& a) {
  return (a.top_k_rows || a.top_k == 0 || a.top_k >= a.vocab) && (a.top_p_rows || a.min_p_rows || a.top_p < 1.0 || a.min_p > 0.0);
}

// Where the parts of the scratch are: a pointer is 0 bytes from its start where there is none.
struct Scratch {
  int64_t seg_s, seg_m, kept_seg, bins, list, info, end;
};
Scratch scratch_of(const DrawArgs& a) {
  const int64_t rows = a.rows, n = rows * segments(a.vocab), binned = may_bin(a) ? rows : 0;
  Scratch s;
  s.seg_s = 0;
  s.kept_seg = s.seg_s + 8 * n;
  s.bins = s.kept_seg + (binned ? 8 * n : 0);
  s.list = s.bins + 8 * binned * BINS;
  s.info = s.list + 8 * binned * LIST;
  s.seg_m = s.info + (int64_t)sizeof(DrawRow) * binned;
  s.end = (s.seg_m + 4 * n + 15) / 16 * 16;
  return s;
}

template <typename T, bool VEC>
hipError_t run(const DrawArgs& a, hipStream_t st) {
  const int segs = segments(a.vocab);
  const int64_t items = (int64_t)a.rows * segs, grid = (items + SCAN_WAVES - 1) / SCAN_WAVES;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  hipError_t e = kv8_launch(k_draw_scan<T, VEC>, dim3((unsigned)grid), dim3(64 * SCAN_WAVES), st, a, segs, items);
  if (e != hipSuccess) return e;
  if (a.bins) {
    const int parts = (int)std::max<int64_t>(1, std::min<int64_t>(1024 / a.rows, (segs + 7) / 8));
    if ((int64_t)a.rows * parts > INT32_MAX) return hipErrorInvalidValue;
    const dim3 g((unsigned)(a.rows * parts));
    if ((e = kv8_launch(k_draw_bins<T, VEC>, g, dim3(PART), st, a, segs, parts)) != hipSuccess) return e;
    if ((e = kv8_launch(k_draw_collect<T, VEC>, g, dim3(PART), st, a, segs, parts)) != hipSuccess) return e;
  }
  return may_cut(a) ? kv8_launch(k_draw_pick<T, VEC, true>, dim3(a.rows), dim3(PICK), st, a, segs)
                    : kv8_launch(k_draw_pick<T, VEC, false>, dim3(a.rows), dim3(PICK), st, a, segs);
}

}  // namespace

int64_t draw_scratch_bytes(const DrawArgs& a) { return scratch_of(a).end; }

hipError_t launch_draw(DrawArgs a, void* scratch, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  if (a.vocab < 1 || a.vocab > DRAW_MAX_VOCAB) return hipErrorInvalidValue;
  const Scratch s = scratch_of(a);
  char* p = (char*)scratch;
  a.seg_s = (double*)(p + s.seg_s);
  a.seg_m = (float*)(p + s.seg_m);
  if (may_bin(a)) {
    a.kept_seg = (unsigned long long*)(p + s.kept_seg);
    a.bins = (unsigned long long*)(p + s.bins);
    a.list = (unsigned long long*)(p + s.list);
    a.info = (DrawRow*)(p + s.info);
  }
  const bool vec = (uintptr_t)a.logits % 16 == 0 && a.row * (a.dtype == 1 ? 2 : 4) % 16 == 0;
  if (a.dtype == 1) return vec ? run<bf16_t, true>(a, st) : run<bf16_t, false>(a, st);
  return vec ? run<float, true>(a, st) : run<float, false>(a, st);
}
