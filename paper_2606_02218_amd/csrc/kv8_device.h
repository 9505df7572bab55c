// Device helpers of the 8-bit key/value cache (gfx950): block addresses, the
// rows of a ragged batch, e4m3 conversions.
#pragma once
#include "rg_device.h"
#include "rg_kernels.h"

#include <hip/hip_ext.h>

// Launches a kernel, timed where the policy's profile asks for it.  Straight
// through hipLaunchKernel: the chevrons' pushed and popped configuration costs a
// quarter of a microsecond of the three that a launch takes the host.  Launches of
// 2^32 threads and more in a dimension, which hipLaunchKernel would wrap without
// an error, are refused here.
template <typename T> struct KernelArg { typedef T type; };
template <typename... Args>
hipError_t kv8_launch(void (*kernel)(Args...), dim3 grid, dim3 block, hipStream_t st, typename KernelArg<Args>::type... args) {
  if ((uint64_t)grid.x * block.x >> 32 || (uint64_t)grid.y * block.y >> 32) return hipErrorInvalidConfiguration;
  void* p[] = {(void*)&args...};
  hipEvent_t e0, e1;
  const hipError_t e = rg_take_launch_events(&e0, &e1)
                           ? hipExtLaunchKernel((const void*)kernel, grid, block, p, 0, st, e0, e1, 0)
                           : hipLaunchKernel((const void*)kernel, grid, block, p, 0, st);
  if (e != hipSuccess) (void)hipGetLastError();   // reported here, not by the next call
  return e;
}

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

// Page table row of sequence s; nullptr when it lies outside the table.
__device__ __forceinline__ const int32_t* kv8_table(const Kv8Rows& b, int s) {
  const int t = b.tab_row ? b.tab_row[s] : s;
  return (unsigned)t < (unsigned)b.tab_rows ? b.tab + (int64_t)t * b.tab_stride : nullptr;
}

// Tokens that a row is taken to see where its length passes the table's
// capacity: one block more than the table holds, which makes the row NaN
// without a walk over what is not there.
__device__ __forceinline__ int kv8_most(const Kv8Pool& c, const Kv8Rows& b) {
  return b.tab_stride * (16 << c.sub_shift) + 16;   // at most 2^30 + 16
}

// Index of the block that holds tokens 16 * blk .. + 15 of a sequence for one
// kv head; -1 where the table has no such page (or the page is none of the
// pool's).
__device__ __forceinline__ int kv8_block(const Kv8Pool& c, const int32_t* tab, int tab_stride, int blk, int kvh) {
  const int slot = blk >> c.sub_shift;
  if (!tab || (unsigned)slot >= (unsigned)tab_stride) return -1;
  const int page = tab[slot];
  if ((unsigned)page >= (unsigned)c.pages) return -1;
  return ((page * c.n_kv + kvh) << c.sub_shift) + (blk & ((1 << c.sub_shift) - 1));
}

// Sequence s of batch b: its first row (clipped to the batch) and row count.
__device__ __forceinline__ void kv8_seq_rows(const Kv8Rows& b, int s, int& r0, int& n) {
  if (!b.seq_off) {
    r0 = s;
    n = s < (b.d_rows ? *b.d_rows : b.rows) ? 1 : 0;
    return;
  }
  r0 = min(max(b.seq_off[s], 0), b.rows);
  n = min(max(b.seq_off[s + 1], r0), b.rows) - r0;
}

// The sequence with the largest key(s) = off(s) / span + per_seq * s not above
// x: work items of `span` rows, numbered through a batch without a pass over
// it, since a sequence never has more items than its keys leave room for.
__device__ __forceinline__ int kv8_find(const Kv8Rows& b, int x, int span, int per_seq, int& key) {
  int lo = 0, hi = b.n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (min(max(b.seq_off[mid], 0), b.rows) / span + per_seq * mid <= x) lo = mid;
    else hi = mid;
  }
  key = min(max(b.seq_off[lo], 0), b.rows) / span + per_seq * lo;
  return lo;
}

// Tokens of sequence s, this call's rows counted; a length below zero is none.
__device__ __forceinline__ int kv8_len(const Kv8Rows& b, int s) { return max(b.seq_len[s] + b.len_add, 0); }

// Largest value of the wave's lanes (none below zero), in every lane: through the
// vector unit's own lane moves, half the latency of six exchanges through LDS.
template <typename T>
__device__ __forceinline__ T wave_max_dpp(T x) {
  static_assert(sizeof(T) == 4, "32 bits a lane");
  int v = __builtin_bit_cast(int, x);         // the order of floats above zero is that of their bits
#define RG_DPP_MAX(ctrl) v = max(v, __builtin_amdgcn_update_dpp(v, v, ctrl, 0xf, 0xf, false))
  RG_DPP_MAX(0x111);   // row_shr 1, 2, 4, 8: lane 15 of each row of 16 has its maximum
  RG_DPP_MAX(0x112);
  RG_DPP_MAX(0x114);
  RG_DPP_MAX(0x118);
  RG_DPP_MAX(0x142);   // row_bcast 15, 31: lane 63 has the wave's
  RG_DPP_MAX(0x143);
#undef RG_DPP_MAX
  return __builtin_bit_cast(T, __builtin_amdgcn_readlane(v, 63));
}

// Sum of the wave's lanes, and the index of the k-th set bit of a wave's mask (one
// that has more than k), in every lane.
__device__ __forceinline__ int wave_sum_dpp(int v) {
#define RG_DPP_ADD(ctrl, rows) v += __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xf, false)
  RG_DPP_ADD(0x111, 0xf);   // row_shr 1, 2, 4, 8: lane 15 of each row of 16 has its sum
  RG_DPP_ADD(0x112, 0xf);
  RG_DPP_ADD(0x114, 0xf);
  RG_DPP_ADD(0x118, 0xf);
  RG_DPP_ADD(0x142, 0xa);   // row_bcast 15 into rows 1 and 3, 31 into rows 2 and 3
  RG_DPP_ADD(0x143, 0xc);
#undef RG_DPP_ADD
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int wave_nth_bit(uint64_t mask, int k) {
  const int lane = threadIdx.x & 63;
  const int below = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
  return __ffsll((unsigned long long)__ballot((mask >> lane & 1) && below == k)) - 1;
}

// Row r of batch b: its sequence and position there (negative: a padding row).
// False for rows of no sequence.
__device__ __forceinline__ bool kv8_row(const Kv8Rows& b, int r, int& s, int& pos) {
  if (!b.seq_off) {
    s = r;
    if (r >= (b.d_rows ? *b.d_rows : b.rows)) return false;
    pos = kv8_len(b, s) - 1;
    return true;
  }
  int key;
  s = kv8_find(b, r, 1, 0, key);
  int r0, n;
  kv8_seq_rows(b, s, r0, n);
  if (r < r0 || r >= r0 + n) return false;
  pos = kv8_len(b, s) - (r0 + n - r);
  return true;
}

// Four e4m3 codes times a power-of-two scale as four bf16 values (exact: a
// code has four significant bits).
__device__ __forceinline__ u32x2_t kv8_bf16x4(uint32_t codes, float scale) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true);
  return u32x2_t{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
}

__device__ __forceinline__ bf16x8_t kv8_bf16x8(uint32_t lo, uint32_t hi, float s_lo, float s_hi) {
  const u32x2_t a = kv8_bf16x4(lo, s_lo), b = kv8_bf16x4(hi, s_hi);
  return __builtin_bit_cast(bf16x8_t, u32x4_t{a[0], a[1], b[0], b[1]});
}

// Nearest e4m3 codes of four values that are scaled already: ties to even,
// magnitudes above 448 (infinities too) become 448, NaN becomes code 255 (NaN).
__device__ __forceinline__ uint32_t kv8_codes4(float a, float b, float c, float d) {
  auto sat = [](float x) { return fabsf(x) > 448.f ? copysignf(448.f, x) : x; };   // false for NaN
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(sat(a), sat(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(sat(c), sat(d), w, true);
  return (uint32_t)w;
}

// Four codes requantized by `ratio` (old scale / new scale).
__device__ __forceinline__ uint32_t kv8_requant4(uint32_t codes, float ratio) {
  const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false);
  const f32x2_t b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  return kv8_codes4(a[0] * ratio, a[1] * ratio, b[0] * ratio, b[1] * ratio);
}

// Block scale of a largest magnitude: 2^k for the least k in [-64, 119] with
// 448 * 2^k >= amax.  448 = 0.875 * 2^9, so k follows from amax's exponent and
// whether its fraction passes 0.875 (1.75 of the stored form): no rounding.
__device__ __forceinline__ float kv8_scale(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int k = (int)(u >> 23) - 126 - ((u & 0x7FFFFFu) <= 0x600000u ? 9 : 8);
  return __uint_as_float((uint32_t)(min(max(k, -64), 119) + 127) << 23);
}

// The two members of a turned pair.  The fused operation is written out, so that
// every variant of a kernel rounds alike.
__device__ __forceinline__ float turn_lo(float a, float b, float c, float s) { return fmaf(a, c, -(b * s)); }
__device__ __forceinline__ float turn_hi(float a, float b, float c, float s) { return fmaf(b, c, a * s); }

// N consecutive elements as fp32: 16-byte loads where VEC, else one by one.
template <int N, bool VEC> __device__ __forceinline__ void ld_elems(const float* p, float (&v)[N]) {
  if constexpr (VEC && N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const f32x4_t x = *reinterpret_cast<const f32x4_t*>(p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + e] = x[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = p[i];
  }
}
template <int N, bool VEC> __device__ __forceinline__ void ld_elems(const bf16_t* p, float (&v)[N]) {
  if constexpr (VEC && N % 8 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t*>(p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[i + 2 * e] = __uint_as_float(x[e] << 16);
        v[i + 2 * e + 1] = __uint_as_float(x[e] & 0xFFFF0000u);
      }
    }
  } else if constexpr (VEC && N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x2_t x = *reinterpret_cast<const u32x2_t*>(p + i);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        v[i + 2 * e] = __uint_as_float(x[e] << 16);
        v[i + 2 * e + 1] = __uint_as_float(x[e] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = bf16_to_f32(p[i]);
  }
}

template <int N, bool VEC> __device__ __forceinline__ void st_elems(float* p, const float (&v)[N]) {
  if constexpr (VEC && N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4_t*>(p + i) = f32x4_t{v[i], v[i + 1], v[i + 2], v[i + 3]};
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = v[i];
  }
}
template <int N, bool VEC> __device__ __forceinline__ void st_elems(bf16_t* p, const float (&v)[N]) {
  if constexpr (VEC && N % 8 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 8)
      *reinterpret_cast<u32x4_t*>(p + i) = u32x4_t{pack_bf16x2(v[i], v[i + 1]), pack_bf16x2(v[i + 2], v[i + 3]),
                                                   pack_bf16x2(v[i + 4], v[i + 5]), pack_bf16x2(v[i + 6], v[i + 7])};
  } else if constexpr (VEC && N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      *reinterpret_cast<u32x2_t*>(p + i) = u32x2_t{pack_bf16x2(v[i], v[i + 1]), pack_bf16x2(v[i + 2], v[i + 3])};
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = (bf16_t)(pack_bf16x2(v[i], 0.f) & 0xFFFFu);
  }
}
