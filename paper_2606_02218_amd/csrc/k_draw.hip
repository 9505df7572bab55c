// Sampling from given logits and given uniform numbers: temperature, top-k, top-p,
// min-p.
//
// Weights are w = exp((z - max z) / T).  Tokens in order of z, ties by id: top-k keeps
// the first k, top-p those before which less than p of the k's weight lies, min-p
// those with z >= max z + T ln(min_p).  Each keeps a beginning of that order, so all
// together keep one: the tokens up to a border (z, id).  The draw is the first token,
// by id, at which the kept weights' running sum passes u times their sum.
//
// Two launches.  The first streams the logits once: maximum and sum of weights of
// every segment of 512 tokens, the sum in fp32 with respect to that maximum.  The
// second, a workgroup a row, finds the border and draws.
// Weights of the kept tokens are whole numbers, w 2^42 to nearest: their sums do not
// depend on any order, so LDS atomics give the same draw on every run.
#include <algorithm>
#include <type_traits>

#include "kv8_device.h"

namespace {

constexpr int SEG = 512;              // tokens of a segment
constexpr int MAX_SEGS = 2048;        // of a row: 2^20 tokens
constexpr int SCAN_WAVES = 4;
constexpr int PICK = 512;             // threads of a row in the second launch
constexpr int BINS = 2 * PICK;        // of weights, 16 an octave
constexpr int LIST = 4096;            // candidates that LDS holds
constexpr int FEW = 64;               // tokens that a wave puts in order, a lane each
constexpr float LOG2E = 1.44269504088896341f;

// Settings of a row.
struct RowOpts {
  float temperature, top_p, min_p;
  int top_k;
};
__device__ __forceinline__ RowOpts row_opts(const DrawArgs& A, int r) {
  RowOpts o;
  o.temperature = A.temperature_rows ? A.temperature_rows[r] : A.temperature;
  o.top_k = A.top_k_rows ? A.top_k_rows[r] : A.top_k;
  o.top_p = A.top_p_rows ? A.top_p_rows[r] : A.top_p;
  o.min_p = A.min_p_rows ? A.min_p_rows[r] : A.min_p;
  return o;
}
// Base-2 exponent of a weight per logit; temperature 0 (the largest logit) reports at 1.
// Tiny temperatures: a finite factor, as 0 times infinity would be NaN.
__device__ __forceinline__ float inv_temperature(float t) { return t == 0.f ? LOG2E : fminf(LOG2E / t, 3.0e38f); }

template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int64_t i, int64_t n, float (&v)[8]) {
  if (VEC && i + 8 <= n) {
    ld_elems<8, true>(p + i, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = i + e < n ? ld_f32<T>(p + i + e) : -INFINITY;
  }
}

// ---------------------------------------------------------------- segments
template <typename T, bool VEC>
__global__ __launch_bounds__(64 * SCAN_WAVES) void k_draw_scan(DrawArgs A, int segs, int64_t items) {
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * SCAN_WAVES + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (item >= items) return;
  const int r = (int)(item / segs), seg = (int)(item - (int64_t)r * segs);
  const float c = inv_temperature(A.temperature_rows ? A.temperature_rows[r] : A.temperature);
  float v[8];
  load8<T, VEC>((const T*)A.logits + r * A.row, (int64_t)seg * SEG + 8 * lane, A.vocab, v);
  float m = v[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) m = fmaxf(m, v[e]);
  m = wave_max(m);
  const float ref = m == -INFINITY ? 0.f : m;     // nothing here: weights exp2(-inf) = 0
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s += __builtin_amdgcn_exp2f((v[e] - ref) * c);
  s = wave_sum(s);
  if (lane == 0) {
    A.seg[2 * item] = m;
    A.seg[2 * item + 1] = s;
  }
}

// ---------------------------------------------------------------- a row
typedef unsigned long long u64;
constexpr double FIXED_ONE = 4398046511104.0;   // 2^42
constexpr int ID_BITS = 20;

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

// w 2^42 of a weight in [0, 1], to nearest.
__device__ __forceinline__ u64 fixed_weight(float w) {
  const uint32_t u = __float_as_uint(w);
  const int e = (int)(u >> 23) - 127 + 19;                      // 42 - 23
  const u64 m = (u & 0x7FFFFFu) | 0x800000u;
  return e >= 0 ? m << e : e < -24 ? 0 : (m + (1ull << (-e - 1))) >> -e;
}

// Over the PICK threads of a row; `red` holds a value a wave.
template <typename V>
__device__ __forceinline__ V row_prefix(V v, V* red, V* total) {   // inclusive
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
  for (int i = 0; i < PICK / 64; ++i) {
    if (i < w) v += red[i];
    all += red[i];
  }
  *total = all;
  return v;
}
__device__ __forceinline__ double row_sum(double v, double* red) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  v = wave_sum_d(v);
  __syncthreads();
  if (lane == 0) red[w] = v;
  __syncthreads();
  double r = 0.0;
#pragma unroll
  for (int i = 0; i < PICK / 64; ++i) r += red[i];
  return r;
}
__device__ __forceinline__ int row_min(int v, int* red) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if (lane == 0) red[w] = v;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PICK / 64; ++i) v = min(v, red[i]);
  return v;
}

struct RowMemory {
  float m[MAX_SEGS], s[MAX_SEGS];     // of the segments
  double red[PICK / 64];
  u64 red64[PICK / 64];
  float redf[16];
  int redi[PICK / 64];
  double start;
};
struct CutMemory {
  union {
    struct { u64 mass[BINS]; uint32_t count[BINS]; } bin;
    u64 seg[MAX_SEGS];                // kept weight of each segment
  };
  u64 list[LIST];                     // places of the tokens that can be kept
  u64 few[FEW];
  u64 found, mass, rank;
  int n_list, n_few;
};

// What a row's threads know of it.
template <typename T, bool VEC>
struct Row {
  const T* z;
  int vocab, segs, top;               // top: the first segment that holds the maximum
  float zmax, c;
  RowMemory* S;

  __device__ float token(int s) const {   // a thread a token of segment s
    const int i = s * SEG + (int)threadIdx.x;
    return i < vocab ? ld_f32<T>(z + i) : -INFINITY;
  }
  __device__ float weight(float x) const { return __builtin_amdgcn_exp2f((x - zmax) * c); }
  __device__ u64 fixed(float x) const { return fixed_weight(weight(x)); }
  // f(z, id) for every token of at least t0; whole waves call it.
  template <typename F>
  __device__ void from_memory(float t0, F f) const {
    for (int s = (int)threadIdx.x >> 6; s < segs; s += PICK / 64) {
      if (S->m[s] < t0) continue;
      float v[8];
      const int i = s * SEG + 8 * ((int)threadIdx.x & 63);
      load8<T, VEC>(z, i, vocab, v);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i + e < vocab && v[e] >= t0) f(v[e], i + e);
    }
  }
};

// The border of top-k (by rank: fewer than `limit` tokens come before) or top-p (less
// than `limit` of weight does): the place of the last token that is kept, 0 if all of
// them are; mass: the weight up to it.  Bins of weight first, then ever finer windows
// of places, until a wave can put what is left in order.
template <typename R, typename Each>
__device__ u64 find_border(const R& row, CutMemory& C, const Each& each, bool by_rank, double limit, u64* mass) {
  const int tid = threadIdx.x;
  auto bin_of = [&](float x) { return (int)fminf((row.zmax - x) * row.c * 16.f, (float)(BINS - 1)); };   // falls as x grows
  u64 rank0 = 0, mass0 = 0;           // before the window
  u64 lo = 0;
  int shift = 64, bin = 0;            // the window: places lo .. lo + 2^shift - 1 of the bin
  for (int level = 0;; ++level) {
    __syncthreads();
    for (int i = tid; i < BINS; i += PICK) { C.bin.mass[i] = 0; C.bin.count[i] = 0; }
    if (tid == 0) C.n_few = 0;
    __syncthreads();
    const int next = level == 0 ? 0 : max(shift - 10, 0);
    each([&](float x, int id) {
      int d;
      if (level == 0) {
        d = bin_of(x);
      } else {
        const u64 p = place_of(x, id);
        if (bin_of(x) != bin || p < lo || (p - lo) >> shift) return;
        d = BINS - 1 - (int)((p - lo) >> next);
      }
      atomicAdd(&C.bin.mass[d], row.fixed(x));
      atomicAdd(&C.bin.count[d], 1u);
    });
    __syncthreads();
    // the first digit whose end reaches the limit
    const u64 m0 = C.bin.mass[2 * tid], m1 = C.bin.mass[2 * tid + 1];
    const uint32_t n0 = C.bin.count[2 * tid], n1 = C.bin.count[2 * tid + 1];
    u64 all_m, all_n;
    const u64 m = row_prefix(m0 + m1, row.S->red64, &all_m) + mass0;
    const u64 n = row_prefix((u64)(n0 + n1), row.S->red64, &all_n) + rank0;
    auto reaches = [&](u64 rank, u64 weight) { return by_rank ? (double)rank >= limit : (double)weight >= limit; };
    int hit = INT32_MAX;
    if (n1 && reaches(n, m)) hit = 2 * tid + 1;
    if (n0 && reaches(n - n1, m - m1)) hit = 2 * tid;
    const int d = row_min(hit, row.S->redi);
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
    const uint32_t inside = C.bin.count[d];
    if (level == 0) {
      bin = d;
      lo = 0;
      shift = 32 + ID_BITS;
    } else {
      lo += (u64)(BINS - 1 - d) << next;
      shift = next;
    }
    if (inside > FEW) continue;       // places differ: at the latest a window of 1 has one token
    each([&](float x, int id) {
      const u64 p = place_of(x, id);
      if (bin_of(x) == bin && p >= lo && !((p - lo) >> shift)) C.few[atomicAdd(&C.n_few, 1)] = p;
    });
    __syncthreads();
    if (tid < 64) {
      const u64 p = tid < (int)inside ? C.few[tid] : 0;
      const u64 w = tid < (int)inside ? row.fixed(z_of(p)) : 0;
      u64 before = mass0, rank = rank0;
      for (int j = 0; j < (int)inside; ++j) {
        const u64 q = C.few[j], v = row.fixed(z_of(q));
        if (q > p) { ++rank; before += v; }
      }
      if (tid < (int)inside && !reaches(rank, before) && reaches(rank + 1, before + w)) { C.found = p; C.mass = before + w; }
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
  const int r = blockIdx.x, tid = threadIdx.x;
  const RowOpts o = row_opts(A, r);
  const float* seg = A.seg + (int64_t)r * segs * 2;
  const double u = A.u64 ? ((const double*)A.u)[r] : (double)((const float*)A.u)[r];
  Row<T, VEC> row{(const T*)A.logits + r * A.row, A.vocab, segs, 0, -INFINITY, inv_temperature(o.temperature), &S};

  float zmax = -INFINITY;
  for (int i = tid; i < segs; i += PICK) {
    S.m[i] = seg[2 * i];
    S.s[i] = seg[2 * i + 1];
    zmax = fmaxf(zmax, S.m[i]);
  }
  row.zmax = zmax = block_max(zmax, S.redf);
  int top = INT32_MAX;
  for (int i = tid; i < segs; i += PICK)
    if (S.m[i] == zmax) top = min(top, i);
  row.top = top = row_min(top, S.redi);
  // The sum of all weights.  That of the segment which holds the maximum is taken
  // again in 64 bits: a weight of 1 beside small ones.
  auto share = [&](int i) { return S.m[i] == -INFINITY ? 0.0 : (double)S.s[i] * (double)row.weight(S.m[i]); };
  double part = 0.0;
  for (int i = tid; i < segs; i += PICK)
    if (i != top) part += share(i);
  const double others = row_sum(part, S.red);
  const double largest = row_sum(top < segs && top * SEG + tid < A.vocab ? (double)row.weight(row.token(top)) : 0.0, S.red);
  const double total = others + largest;

  // NaN logits make the total NaN, as does an infinite maximum
  const bool good = zmax > -INFINITY && zmax < INFINITY && total < INFINITY && o.temperature >= 0.f &&
                    o.temperature < INFINITY && u >= 0.0 && u < 1.0 && o.top_p == o.top_p && o.min_p == o.min_p;
  if (!good) {
    if (tid == 0) {
      A.token[r] = -1;
      A.logprob[r] = A.kept[r] = __uint_as_float(0x7FC00000u);
    }
    return;
  }
  const double inv_t = o.temperature == 0.f ? 1.0 : 1.0 / (double)o.temperature;
  auto answer = [&](int id, float zi, double log_kept) {
    const double lw = ((double)zi - (double)zmax) * inv_t;
    A.token[r] = id;
    A.logprob[r] = (float)(lw - log(total));
    A.kept[r] = (float)(o.temperature == 0.f ? 0.0 : lw - log_kept);
  };
  // The token of segment s at which the running sum, `before` in front of it, passes
  // `want`; w is the weight of the thread's token.
  auto finish = [&](int s, float zi, auto w, auto before, double want, double log_kept) {
    decltype(w) all;
    const auto incl = row_prefix(w, reinterpret_cast<decltype(w)*>(S.red64), &all) + before;
    int hit = row_min(w > 0 && (double)incl > want ? tid : INT32_MAX, S.redi);
    if (hit == INT32_MAX) hit = -row_min(w > 0 ? -tid : 1, S.redi);   // roundings next to u = 1: the last with a weight
    if (tid == hit) answer(s * SEG + tid, zi, log_kept);
  };
  // The first segment at whose end the running sum of f(segment) passes `want`, and the
  // sum in front of it.
  auto find_segment = [&](auto f, double want, auto& before) {
    using V = typename std::remove_reference<decltype(before)>::type;
    V run = 0;
    for (int base = 0; base < segs; base += PICK) {
      const int i = base + tid;
      const V w = i < segs ? f(i) : 0;
      V all;
      const V incl = row_prefix(w, reinterpret_cast<V*>(S.red64), &all) + run;
      const int at = row_min(w > 0 && (double)incl > want ? i : INT32_MAX, S.redi);
      if (at != INT32_MAX) {
        if (i == at) *reinterpret_cast<V*>(&S.start) = incl - w;
        __syncthreads();
        before = *reinterpret_cast<V*>(&S.start);
        return at;
      }
      run += all;
    }
    before = 0;
    return top;
  };

  if (o.temperature == 0.f) {         // the first of the largest
    const float zi = row.token(top);
    const int at = row_min(zi == zmax ? tid : INT32_MAX, S.redi);
    if (tid == at) answer(top * SEG + tid, zi, 0.0);
    return;
  }
  const bool by_k = o.top_k > 0 && o.top_k < A.vocab, by_p = o.top_p < 1.f, by_min = o.min_p > 0.f;
  if (!CUT || !(by_k || by_p || by_min)) {   // every token can be drawn
    double before;
    const int at = find_segment([&](int i) { return i == top ? largest : share(i); }, u * total, before);
    const float zi = row.token(at);
    finish(at, zi, (double)row.weight(zi), before, u * total, log(total));
    return;
  }
  if constexpr (CUT) {
    CutMemory* const C = &cut;
    float t0 = -INFINITY;             // no token below it is kept
    u64 border = 0;
    if (by_min) {                     // the least fp32 value that is not below max z + T ln(min_p)
      const double lowest = (double)zmax + (double)o.temperature * log(fmin((double)o.min_p, 1.0));
      float t = (float)lowest;
      if ((double)t < lowest) t = of_key(key_of(t) + 1);
      border = (u64)key_of(t) << ID_BITS;
      if (!by_k || !by_p) t0 = t;     // top-p takes its share of all the k
    }
    if (tid == 0) C->n_list = 0;
    __syncthreads();
    row.from_memory(t0, [&](float x, int id) {
      const int n = atomicAdd(&C->n_list, 1);
      if (n < LIST) C->list[n] = place_of(x, id);
    });
    __syncthreads();
    const int n_list = C->n_list;
    auto each = [&](auto f) {
      if (n_list <= LIST) {
        for (int i = tid; i < n_list; i += PICK) f(z_of(C->list[i]), id_of(C->list[i]));
      } else {
        row.from_memory(t0, f);
      }
    };
    double all = total * FIXED_ONE;
    if (by_k) {
      u64 mass;
      border = max(border, find_border(row, *C, each, true, (double)o.top_k, &mass));
      all = (double)mass;
    }
    if (by_p) {
      u64 mass;
      border = max(border, find_border(row, *C, each, false, fmax((double)o.top_p * all, 0.5), &mass));
    }
    __syncthreads();
    for (int i = tid; i < MAX_SEGS; i += PICK) C->seg[i] = 0;
    __syncthreads();
    each([&](float x, int id) {
      if (place_of(x, id) >= border) atomicAdd(&C->seg[id / SEG], row.fixed(x));
    });
    __syncthreads();
    u64 mine = 0, kept, before;
    for (int i = tid; i < segs; i += PICK) mine += C->seg[i];
    row_prefix(mine, S.red64, &kept);
    const int at = find_segment([&](int i) { return C->seg[i]; }, u * (double)kept, before);
    const float zi = row.token(at);
    const int id = at * SEG + tid;
    finish(at, zi, id < A.vocab && place_of(zi, id) >= border ? row.fixed(zi) : (u64)0, before, u * (double)kept,
           log((double)kept / FIXED_ONE));
  }
}

int segments(int vocab) { return (vocab + SEG - 1) / SEG; }

template <typename T, bool VEC>
hipError_t run(const DrawArgs& a, hipStream_t st) {
  const int segs = segments(a.vocab);
  const int64_t items = (int64_t)a.rows * segs, grid = (items + SCAN_WAVES - 1) / SCAN_WAVES;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  const hipError_t e = kv8_launch(k_draw_scan<T, VEC>, dim3((unsigned)grid), dim3(64 * SCAN_WAVES), st, a, segs, items);
  if (e != hipSuccess) return e;
  const bool cut = a.top_k_rows || a.top_p_rows || a.min_p_rows || a.top_k > 0 || a.top_p < 1.f || a.min_p > 0.f;
  return cut ? kv8_launch(k_draw_pick<T, VEC, true>, dim3(a.rows), dim3(PICK), st, a, segs)
             : kv8_launch(k_draw_pick<T, VEC, false>, dim3(a.rows), dim3(PICK), st, a, segs);
}

}  // namespace

int64_t draw_scratch_floats(int64_t rows, int vocab) { return 2 * rows * segments(vocab); }

hipError_t launch_draw(const DrawArgs& a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  if (a.vocab < 1 || a.vocab > DRAW_MAX_VOCAB) return hipErrorInvalidValue;
  const bool vec = (uintptr_t)a.logits % 16 == 0 && a.row * (a.dtype == 1 ? 2 : 4) % 16 == 0;
  if (a.dtype == 1) return vec ? run<bf16_t, true>(a, st) : run<bf16_t, false>(a, st);
  return vec ? run<float, true>(a, st) : run<float, false>(a, st);
}
