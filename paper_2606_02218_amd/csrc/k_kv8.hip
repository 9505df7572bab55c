// Append to the 8-bit key/value cache: rotate the keys, quantize keys and
// values by block, write both into their pages, and rotate the queries on the
// way.
//
// A block is 16 consecutive tokens of one kv head.  Its scale is the power of
// two s = 2^k with the least k for which the largest magnitude of its rows fits
// e4m3 (448 s), never below the scale of tokens that stay in it; a code is
// x / s rounded to nearest even.  The scale being a power of two, x / s is exact,
// an e4m3 code keeps the same four bits under every scale that holds it, and
// tokens that stay lose bits only where a grown scale pushes them among the
// subnormal codes.
//
// One wave owns a block of keys or of values from load to store, so nothing of
// a block is shared between waves and no order matters.  Keys: four lanes a
// token, a 16-dim granule each at a time, stored as the 16 bytes the attention
// loads.  Values: a lane takes 4 tokens of a few dims, whose codes are the
// stored dwords.  Queries: a wave a row.  Bound by memory for prompts (32 of 512
// tokens, 4 kv and 28 query heads of 128 in bf16, 294 MB: 58 us, 5.1 TB/s), by the
// chain position -> page -> scale -> store for single tokens (512 rows of 2 kv and
// 12 query heads 6.5 us, 8 rows 5.2).
#include <algorithm>

#include "kv8_device.h"
#include "rope_device.h"

namespace {

struct AppendArgs {
  Kv8Pool c;
  Kv8Rows b;
  HeadView k, v, q;
  HeadOut q_out;
  int n_q;
  RopeTable t;
  unsigned blocks;   // block items: bound on the batch's blocks x n_kv x 2
};

__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;   // NaN and infinities do not set a scale
}

// Dims d0 .. d0 + 7 of a key, turned.  x: the head; ok: the position is in the table.
template <typename T, bool VEC, int LAYOUT>
__device__ __forceinline__ void turned8(const T* x, int d0, const RopeTable& t, const float* co, const float* si, bool ok,
                                        float (&y)[8]) {
  ld_elems<8, VEC>(x + d0, y);
  const int m = t.pairs;
  if (d0 >= 2 * m) return;
  if constexpr (VEC && LAYOUT == 0) {        // m and d0 are multiples of 8: one half or the other
    const bool up = d0 >= m;
    const int i0 = up ? d0 - m : d0;
    float o[8], c[8], s[8];
    ld_elems<8, true>(x + (up ? i0 : d0 + m), o);
    ld_elems<8, true>(co + i0, c);
    ld_elems<8, true>(si + i0, s);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = up ? turn_hi(o[i], y[i], c[i], s[i]) : turn_lo(y[i], o[i], c[i], s[i]);
  } else if constexpr (VEC) {                // 2m is a multiple of 8
    float c[4], s[4];
    ld_elems<4, true>(co + d0 / 2, c);
    ld_elems<4, true>(si + d0 / 2, s);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float a = y[i], b = y[i + 1];
      y[i] = turn_lo(a, b, c[i / 2], s[i / 2]);
      y[i + 1] = turn_hi(a, b, c[i / 2], s[i / 2]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int d = d0 + i;
      if (d >= 2 * m) continue;
      const bool up = LAYOUT ? d & 1 : d >= m;
      const int p = LAYOUT ? d >> 1 : (up ? d - m : d);
      const float o = ld_f32<T>(x + (LAYOUT ? d ^ 1 : (up ? d - m : d + m)));
      y[i] = up ? turn_hi(o, y[i], co[p], si[p]) : turn_lo(y[i], o, co[p], si[p]);
    }
  }
  if (!ok) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (d0 + i < 2 * m) y[i] = __uint_as_float(0x7FC00000u);
  }
}

template <typename T, bool VEC, int LAYOUT, int HD>
__global__ __launch_bounds__(256) void k_kv8_append(AppendArgs A) {
  const int lane = threadIdx.x & 63;
  const unsigned item = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const Kv8Rows& b = A.b;
  if (item >= A.blocks) {                     // a query row
    const int64_t r = item - A.blocks;
    if (r >= b.rows) return;
    int s, pos;
    if (!kv8_row(b, (int)r, s, pos) || pos < 0) return;
    rope_row<T, VEC ? (int)(16 / sizeof(T)) : 1, LAYOUT>((const T*)A.q.p + r * A.q.row, A.q.head,
                                                          (T*)A.q_out.p + r * A.q_out.row, A.q_out.head, A.n_q, HD, A.t,
                                                          pos, 1.f, lane);
    return;
  }
  const bool values = item & 1;
  const unsigned hb = item >> 1;
  const int x = (int)(hb / (unsigned)A.c.n_kv), kvh = (int)(hb - (unsigned)x * A.c.n_kv);
  // item x of the batch: sequence s, its j-th block.  A sequence of n rows
  // touches at most n / 16 + 2 blocks.
  int s = x, key = x, r0, n;
  if (b.seq_off) s = kv8_find(b, x, 16, 2, key);
  kv8_seq_rows(b, s, r0, n);
  if (n <= 0) return;
  const int len = kv8_len(b, s);
  int p0 = len - n;                           // position of row r0
  if (p0 < 0) { r0 -= p0; p0 = 0; }           // padding rows come first
  if (len <= p0) return;
  const int blk = (p0 >> 4) + (x - key);
  if (x < key || blk > (len - 1) >> 4) return;   // x < key: offsets that do not start at 0
  // The chain to the block's address and old scale (page, scale) runs beside the
  // rows' own loads; positions past the table end here.
  const int tr = b.tab_row ? b.tab_row[s] : s, slot = blk >> A.c.sub_shift;
  if ((unsigned)tr >= (unsigned)b.tab_rows || slot >= b.tab_stride) return;
  const int page = b.tab[(int64_t)tr * b.tab_stride + slot];
  const int first = max(p0 - blk * 16, 0), last = min(len - blk * 16, 16);   // the block's new tokens
  const int64_t row0 = (int64_t)r0 + (blk * 16 - p0);                        // row of the block's token 0
  int id = -1;
  float s_old = 0.f;
  float* sp = nullptr;
  uint8_t* out = nullptr;
  auto place = [&]() {                        // false: no such page, nothing to write to
    if ((unsigned)page >= (unsigned)A.c.pages) return false;
    id = ((page * A.c.n_kv + kvh) << A.c.sub_shift) + (blk & ((1 << A.c.sub_shift) - 1));
    sp = (values ? A.c.v_scale : A.c.k_scale) + id;
    out = (values ? A.c.v : A.c.k) + (int64_t)id * (16 * HD);
    if (first > 0) s_old = *sp;
    return true;
  };
  if (!values) {
    constexpr int NG = HD / 64;               // granules of a lane
    const int t = lane >> 2, c = lane & 3;
    const bool fresh = t >= first && t < last;
    float y[2 * NG][8];
    float amax = 0.f;
    if (fresh) {
      const T* kp = (const T*)A.k.p + (row0 + t) * A.k.row + kvh * A.k.head;
      const int pos = blk * 16 + t;
      const bool ok = pos < A.t.n_pos;
      const int64_t to = (int64_t)(ok ? pos : 0) * A.t.pairs;
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          turned8<T, VEC, LAYOUT>(kp, 16 * (c + 4 * g) + 8 * h, A.t, A.t.cos + to, A.t.sin + to, ok, y[2 * g + h]);
    }
    if (!place()) return;
    if (fresh) {
#pragma unroll
      for (int g = 0; g < 2 * NG; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, finite_abs(y[g][i]));
    }
    const float scale = fmaxf(kv8_scale(wave_max_dpp(amax)), s_old), inv = 1.0f / scale;
    if (fresh) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        u32x4_t w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float* z = &y[2 * g + e / 2][4 * (e & 1)];
          w[e] = kv8_codes4(z[0] * inv, z[1] * inv, z[2] * inv, z[3] * inv);
        }
        *reinterpret_cast<u32x4_t*>(out + (c + 4 * g) * 256 + t * 16) = w;
      }
    } else if (t < first && scale > s_old) {
      const float ratio = s_old * inv;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        u32x4_t* w = reinterpret_cast<u32x4_t*>(out + (c + 4 * g) * 256 + t * 16);
        u32x4_t o = *w;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = kv8_requant4(o[e], ratio);
        *w = o;
      }
    }
    if (lane == 0) *sp = scale;
  } else {
    constexpr int DV = HD / 16;               // dims of a lane
    const int tg = lane >> 4, d0 = (lane & 15) * DV;
    float y[4][DV];
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 4 * tg + i;
      if (t >= first && t < last) {
        ld_elems<DV, VEC>((const T*)A.v.p + (row0 + t) * A.v.row + kvh * A.v.head + d0, y[i]);
      } else {
#pragma unroll
        for (int d = 0; d < DV; ++d) y[i][d] = 0.f;
      }
    }
    if (!place()) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = 0; d < DV; ++d) amax = fmaxf(amax, finite_abs(y[i][d]));
    const float scale = fmaxf(kv8_scale(wave_max_dpp(amax)), s_old), inv = 1.0f / scale;
    const bool grown = first > 0 && scale > s_old;
    uint32_t fresh = 0, stay = 0;             // byte masks of the lane's tokens
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 4 * tg + i;
      if (t >= first && t < last) fresh |= 0xFFu << (8 * i);
      if (t < first) stay |= 0xFFu << (8 * i);
    }
    if (fresh || (grown && stay)) {
      uint32_t* w = reinterpret_cast<uint32_t*>(out + tg * 4 * HD + d0 * 4);
      uint32_t o[DV];
      if (fresh != 0xFFFFFFFFu) {
#pragma unroll
        for (int d = 0; d < DV; d += 4) {
          const u32x4_t z = *reinterpret_cast<const u32x4_t*>(w + d);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[d + e] = z[e];
        }
        if (grown && stay) {
          const float ratio = s_old * inv;
#pragma unroll
          for (int d = 0; d < DV; ++d) o[d] = (kv8_requant4(o[d], ratio) & stay) | (o[d] & ~stay);
        }
      } else {
#pragma unroll
        for (int d = 0; d < DV; ++d) o[d] = 0;
      }
#pragma unroll
      for (int d = 0; d < DV; ++d)
        o[d] = (kv8_codes4(y[0][d] * inv, y[1][d] * inv, y[2][d] * inv, y[3][d] * inv) & fresh) | (o[d] & ~fresh);
#pragma unroll
      for (int d = 0; d < DV; d += 4) *reinterpret_cast<u32x4_t*>(w + d) = u32x4_t{o[d], o[d + 1], o[d + 2], o[d + 3]};
    }
    if (lane == 0) *sp = scale;
  }
}

__global__ __launch_bounds__(256) void k_kv8_runs(const int32_t* __restrict__ coff, const int32_t* __restrict__ plen,
                                                  const int32_t* __restrict__ seq_grp, int n_seq, int row0, int n,
                                                  int32_t* __restrict__ off, int32_t* __restrict__ len) {
  const int s = blockIdx.x * blockDim.x + threadIdx.x;
  if (s > n_seq) return;
  const int f = coff[s];
  off[s] = min(max(f - row0, 0), n);
  if (s < n_seq) len[s] = plen[seq_grp[s]] + max(min(coff[s + 1], row0 + n) - f, 0);
}

// Grid (layers, pairs): a workgroup copies one layer of a page.
__global__ __launch_bounds__(256) void k_kv8_page_copy(Kv8Pool c, int64_t layer_blocks, const int32_t* __restrict__ pairs,
                                                       const int32_t* __restrict__ state) {
  const int k = blockIdx.y;
  if (k >= state[3]) return;
  const int64_t n = (int64_t)c.n_kv << c.sub_shift, l0 = blockIdx.x * layer_blocks;   // blocks of a page
  const int64_t src = l0 + pairs[2 * k] * n, dst = l0 + pairs[2 * k + 1] * n;
  const int64_t pieces = n * c.hd;                  // of 16 bytes
  for (int64_t i = threadIdx.x; i < pieces; i += blockDim.x) {
    reinterpret_cast<u32x4_t*>(c.k)[dst * c.hd + i] = reinterpret_cast<const u32x4_t*>(c.k)[src * c.hd + i];
    reinterpret_cast<u32x4_t*>(c.v)[dst * c.hd + i] = reinterpret_cast<const u32x4_t*>(c.v)[src * c.hd + i];
  }
  for (int64_t i = threadIdx.x; i < n; i += blockDim.x) {
    c.k_scale[dst + i] = c.k_scale[src + i];
    c.v_scale[dst + i] = c.v_scale[src + i];
  }
}

bool views_vector(int dtype, const HeadView& x) {
  const int e = dtype == 1 ? 8 : 4;
  return !x.p || ((uintptr_t)x.p % 16 == 0 && x.row % e == 0 && x.head % e == 0);
}

}  // namespace

hipError_t launch_kv8_append(int dtype, const Kv8Pool& c, const Kv8Rows& b, HeadView k, HeadView v, HeadView q,
                             HeadOut q_out, int n_q, const RopeTable& t, hipStream_t st) {
  if (b.rows <= 0 || b.n_seqs <= 0) return hipSuccess;
  if (c.hd != 64 && c.hd != 128) return hipErrorInvalidValue;
  const int64_t items = b.seq_off ? (int64_t)b.rows / 16 + 2 * (int64_t)b.n_seqs : b.n_seqs;
  const int64_t blocks = items * c.n_kv * 2, grid = (blocks + (q.p ? b.rows : 0) + 3) / 4;
  if (grid > (1 << 29)) return hipErrorInvalidValue;   // items are numbered in 32 bits
  const AppendArgs a{c, b, k, v, q, q_out, n_q, t, (unsigned)blocks};
  // whole 16-byte pieces: keys are turned 8 dims at a time
  const bool vec = views_vector(dtype, k) && views_vector(dtype, v) && views_vector(dtype, q) &&
                   views_vector(dtype, HeadView{q_out.p, q_out.row, q_out.head}) &&
                   (t.layout ? (2 * t.pairs) % 8 == 0 : t.pairs % 8 == 0) &&
                   (uintptr_t)t.cos % 16 == 0 && (uintptr_t)t.sin % 16 == 0;
#define RG_APP(T, VEC, LAY, HD) return kv8_launch(k_kv8_append<T, VEC, LAY, HD>, dim3((unsigned)grid), dim3(256), st, a)
#define RG_APP_HD(T, VEC, LAY) \
  if (c.hd == 128) { RG_APP(T, VEC, LAY, 128); } else { RG_APP(T, VEC, LAY, 64); }
#define RG_APP_L(T, VEC) \
  if (t.layout) { RG_APP_HD(T, VEC, 1); } else { RG_APP_HD(T, VEC, 0); }
  if (dtype == 1) {
    if (vec) { RG_APP_L(bf16_t, true); } else { RG_APP_L(bf16_t, false); }
  } else {
    if (vec) { RG_APP_L(float, true); } else { RG_APP_L(float, false); }
  }
#undef RG_APP_L
#undef RG_APP_HD
#undef RG_APP
}

hipError_t launch_kv8_runs(const int32_t* coff, const int32_t* plen, const int32_t* seq_grp, int n_seq, int row0, int n,
                           int32_t* off, int32_t* len, hipStream_t st) {
  hipLaunchKernelGGL(k_kv8_runs, dim3((n_seq + 256) / 256), dim3(256), 0, st, coff, plen, seq_grp, n_seq, row0, n, off,
                     len);
  return hipGetLastError();
}

hipError_t launch_kv8_page_copy(const Kv8Pool& c, int n_layers, int64_t layer_blocks, const int32_t* copy_pairs,
                                int max_pairs, const int32_t* state, hipStream_t st) {
  if (max_pairs <= 0) return hipSuccess;
  hipLaunchKernelGGL(k_kv8_page_copy, dim3(n_layers, max_pairs), dim3(256), 0, st, c, layer_blocks, copy_pairs, state);
  return hipGetLastError();
}
