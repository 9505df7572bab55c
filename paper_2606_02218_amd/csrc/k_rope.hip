// Rotary positions.  Pair i of a head, (a, b) = (x[i], x[i + m]) or
// (x[2i], x[2i + 1]) with m pairs, turns by its position's angle:
//   a' = a cos - b sin,  b' = b cos + a sin,
// with cos and sin of a table, made in 64 bits, that all heads of a row share.
// Dims past 2m are copied.  The gradient with respect to x is the turn back:
// the same with -sin.
//
// Bound by memory: each value is read and written once.  A wave takes one row,
// so its position and table rows are found once; a lane keeps its pairs' cos and
// sin for every head it turns and has four heads' loads in flight.  16384 rows of
// 28 x 128 bf16 (243 MB in and out): 45 us, 5.4 TB/s, where a large copy reaches
// 5.5; 8 rows of 12 x 64: 2.1 us.
#include <algorithm>

#include "kv8_device.h"
#include "rope_device.h"

namespace {

template <typename T, int VEC, int LAYOUT>
__global__ __launch_bounds__(256) void k_rope(const T* x, int64_t x_row, int64_t x_head, T* y, int64_t y_row,
                                              int64_t y_head, const int32_t* __restrict__ pos, int rows, int heads,
                                              int hd, RopeTable t, float sign) {
  const unsigned r = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (r >= (unsigned)rows) return;
  rope_row<T, VEC, LAYOUT>(x + r * x_row, x_head, y + r * y_row, y_head, heads, hd, t, pos[r], sign, threadIdx.x & 63);
}

__global__ void k_rope_table(float* __restrict__ co, float* __restrict__ si, int n_pos, RopeFreqs f) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= (int64_t)n_pos * f.pairs) return;
  const int p = (int)(i / f.pairs), k = (int)(i % f.pairs);
  const double dims = 2.0 * f.pairs;
  double theta = f.theta, amp = 1.0;
  if (f.mode == 2) theta *= pow(f.factor, dims / (dims - 2.0));
  double w = pow(theta, -2.0 * k / dims);
  if (f.mode == 1) w /= f.factor;
  if (f.mode == 3) {
    const double turns = w * f.length / 6.283185307179586476925;
    const double keep = fmin(1.0, fmax(0.0, (turns - f.slow) / (f.fast - f.slow)));
    w *= keep + (1.0 - keep) / f.factor;
    amp = 0.1 * log(f.factor) + 1.0;
  }
  const double a = (double)p * w;
  co[i] = (float)(amp * cos(a));
  si[i] = (float)(amp * sin(a));
}

}  // namespace

hipError_t launch_rope_table(float* co, float* si, int n_pos, const RopeFreqs& f, hipStream_t st) {
  const int64_t n = (int64_t)n_pos * f.pairs;
  if (n < 1 || (n + 255) / 256 > INT32_MAX) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_rope_table, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, co, si, n_pos, f);
  return hipGetLastError();
}

hipError_t launch_rope(int dtype, HeadView x, HeadOut y, const int32_t* pos, int rows, int heads, int hd,
                       const RopeTable& t, bool inverse, hipStream_t st) {
  if (rows <= 0 || heads <= 0) return hipSuccess;
  const float sign = inverse ? -1.f : 1.f;
  constexpr int most = 1 << 25;   // rows of a launch, whose threads have to stay below 2^32
  if (rows > most) {
    const int eb = dtype == 1 ? 2 : 4;
    for (int64_t r = 0; r < rows; r += most) {
      const hipError_t e = launch_rope(dtype, HeadView{(const char*)x.p + r * x.row * eb, x.row, x.head},
                                       HeadOut{(char*)y.p + r * y.row * eb, y.row, y.head}, pos + r,
                                       (int)std::min<int64_t>(most, rows - r), heads, hd, t, inverse, st);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  const dim3 grid(((unsigned)rows + 3) / 4);
  const bool vec = rope_vectors(dtype, x, hd, t) && rope_vectors(dtype, HeadView{y.p, y.row, y.head}, hd, t);
#define RG_ROPE(T, VEC, LAY)                                                                                          \
  return kv8_launch(k_rope<T, VEC, LAY>, grid, dim3(256), st, (const T*)x.p, x.row, x.head, (T*)y.p, y.row, y.head,   \
                    pos, rows, heads, hd, t, sign)
#define RG_ROPE_L(T, VEC) \
  if (t.layout) RG_ROPE(T, VEC, 1); else RG_ROPE(T, VEC, 0)
  if (dtype == 1) {
    if (vec) { RG_ROPE_L(bf16_t, 8); }
    else { RG_ROPE_L(bf16_t, 1); }
  } else {
    if (vec) { RG_ROPE_L(float, 4); }
    else { RG_ROPE_L(float, 1); }
  }
#undef RG_ROPE_L
#undef RG_ROPE
}
