// What the attention passes over the 8-bit key/value cache share: matrix operands
// of queries and probabilities, NaN codes.
#pragma once
#include "kv8_device.h"

constexpr float KV8_SLACK = 8.f;    // the running maximum may lag by 2^8 before accumulators are rescaled
constexpr float KV8_LOG2E = 1.44269504088896341f;
constexpr uint32_t KV8_NAN4 = 0x7F7F7F7Fu;

// Eight fp32 values as N bf16 operands whose sum they are: rounded, then what
// rounding left (8, 17 or all 24 bits; each difference is exact in fp32).  LARGE:
// values that would round past bf16's largest start with that one instead (what is
// left of infinities and NaN becomes NaN in the third piece).
template <int N, bool LARGE = false>
__device__ __forceinline__ void operand8(const float* v, bf16x8_t (&out)[N]) {
  constexpr float top = 3.38953139e38f;       // 2^128 - 2^120
  uint32_t w[N][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = v[2 * i], b = v[2 * i + 1];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (LARGE && n == 0)
        w[n][i] = pack_bf16x2(__builtin_amdgcn_fmed3f(a, -top, top), __builtin_amdgcn_fmed3f(b, -top, top));
      else
        w[n][i] = pack_bf16x2(a, b);
      if (n + 1 < N) {
        a -= __uint_as_float(w[n][i] << 16);
        b -= __uint_as_float(w[n][i] & 0xFFFF0000u);
      }
    }
  }
#pragma unroll
  for (int n = 0; n < N; ++n) out[n] = __builtin_bit_cast(bf16x8_t, u32x4_t{w[n][0], w[n][1], w[n][2], w[n][3]});
}

// Query operand: 8 dims of a row's head.
template <typename T, int N>
__device__ __forceinline__ void query8(const T* p, bool valid, bool vec, bf16x8_t (&out)[N]) {
  float v[8];
  if (!valid) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
  } else if (vec) {
    ld_elems<8, true>(p, v);
  } else {
    ld_elems<8, false>(p, v);
  }
  operand8<N, N == 3>(v, out);
}

__device__ __forceinline__ bool has_nan_code(uint32_t w) { return (((w & KV8_NAN4) + 0x01010101u) & 0x80808080u) != 0; }

// Four codes with NaN ones cleared.
__device__ __forceinline__ uint32_t clear_nan(uint32_t w) {
  const uint32_t hit = (((w & KV8_NAN4) + 0x01010101u) & 0x80808080u) >> 7;
  return w & ~(hit * 0xFFu);
}
