// Causal attention over the 8-bit key/value cache.
//
// Row r of a sequence, at position p, gets per query head
//   o = sum_{j <= p} softmax_j(scale q . k_j) v_j,  k_j, v_j = code * block scale,
// in one pass over the tokens with the running maximum and sum of the softmax.
// Codes become bf16 exactly (four significant bits, power-of-two scales) right
// before the matrix instructions; scores, sums and outputs are fp32.  bf16
// queries are operands as they are.  fp32 values enter as bf16 pieces: three for
// fp32 queries and their probabilities (all 24 bits), two inside a policy (17
// bits, as its other products), two for the probabilities of single bf16 rows,
// where memory leaves the matrix units idle, and one (8 bits, as the output's) for
// runs of bf16 rows, which they bound.
//
// Scores are formed transposed, S^T = K Q^T: tokens are the rows of the
// product, query heads its columns, and a lane ends up with the probabilities of
// one query for just those tokens whose V^T operand it loads.  Nothing moves
// between lanes but the maxima and sums.
//
// * Rows pass (single tokens): a workgroup per row, kv head and context chunk.
//   Its four waves take 32-token steps in turn straight from memory, 16 bytes a
//   lane, and join in LDS.  Bound by the cache's bytes.
// * Tiles pass (runs of rows): a workgroup per 128 query rows (positions x heads
//   of a kv head) and chunk.  64-token pieces of codes go through LDS once for the
//   four waves of 32 query rows.  Bound by the matrix products and, beside them,
//   the exponentials and conversions of the vector units.
// * With several chunks a row, a merge joins their partial results in order.
#include <algorithm>

#include "kv8_device.h"
#include <hip/hip_ext.h>

namespace {

constexpr float KV8_SLACK = 8.f;    // the running maximum may lag by 2^8 before accumulators are rescaled
constexpr float KV8_LOG2E = 1.44269504088896341f;
constexpr uint32_t KV8_NAN4 = 0x7F7F7F7Fu;
constexpr int KV8_TILE_Q = 128;     // query rows of a tile
constexpr int KV8_WAVES = 4;

enum { OUT_F32 = 0, OUT_BF16 = 1, OUT_PLANES = 2 };

// bf16 pieces of a query, and of a probability in either pass.
constexpr int q_pieces(int out) { return out == OUT_F32 ? 3 : out == OUT_PLANES ? 2 : 1; }
constexpr int p_pieces(int out, bool tiles) { return out == OUT_F32 ? 3 : out == OUT_PLANES || !tiles ? 2 : 1; }

// Eight fp32 values as N bf16 operands whose sum they are: rounded, then what
// rounding left (8, 17 or all 24 bits; each difference is exact in fp32).
template <int N>
__device__ __forceinline__ void operand8(const float* v, bf16x8_t (&out)[N]) {
  uint32_t w[N][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = v[2 * i], b = v[2 * i + 1];
#pragma unroll
    for (int n = 0; n < N; ++n) {
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
  operand8<N>(v, out);
}

// N consecutive outputs of (row, head) from dim d on.
template <int OUT, int N>
__device__ __forceinline__ void put(const Kv8Attn& A, int64_t row, int head, int d, const float (&v)[N]) {
  const int64_t at = (row * A.n_q + head) * A.c.hd + d;
  if constexpr (OUT == OUT_F32) {
    st_elems<N, true>((float*)A.out + at, v);
  } else if constexpr (OUT == OUT_BF16) {
    st_elems<N, true>((bf16_t*)A.out + at, v);
  } else {
    float lo[N];
#pragma unroll
    for (int i = 0; i < N; ++i) lo[i] = v[i] - __uint_as_float(pack_bf16x2(v[i], 0.f) << 16);
    st_elems<N, true>((bf16_t*)A.out + at, v);
    st_elems<N, true>((bf16_t*)A.out + A.plane + at, lo);
  }
}

template <int N>
__device__ __forceinline__ void put_part(const Kv8Attn& A, int64_t slot, int head, int d, const float (&v)[N]) {
  st_elems<N, true>(A.part_o + (slot * A.n_q + head) * A.c.hd + d, v);
}
__device__ __forceinline__ float* part_ml(const Kv8Attn& A, int64_t slot, int head) {
  return A.part_ml + (slot * A.n_q + head) * 2;
}

// ---------------------------------------------------------------- rows pass
template <typename T, int HD, int OUT>
__global__ __launch_bounds__(64 * KV8_WAVES) void k_kv8_rows(Kv8Attn A, int htiles, int per_xcd, int64_t items) {
  constexpr int QP = q_pieces(OUT), PP = p_pieces(OUT, false);
  constexpr int NJ = HD / 64;       // 16-byte loads of a block per lane
  constexpr int LDO = HD + 4;
  __shared__ __attribute__((aligned(16))) float sO[KV8_WAVES][16][LDO];
  __shared__ float sM[KV8_WAVES][16], sL[KV8_WAVES][16];

  // Blocks are dealt to the 8 XCDs in turn: neighbouring rows, which share
  // pages where they are siblings of a prompt, go to the same one.
  int64_t item = (int64_t)(blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (item >= items) return;
  const int split = (int)(item % A.plan.n_split);
  item /= A.plan.n_split;
  const int ht = (int)(item % htiles);
  item /= htiles;
  const int kvh = (int)(item % A.c.n_kv), r = (int)(item / A.c.n_kv);
  const int rep = A.n_q / A.c.n_kv, nh = min(16, rep - ht * 16), head0 = kvh * rep + ht * 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  int s, pos;
  if (!kv8_row(A.b, r, s, pos)) return;
  if (pos < 0) {                    // a padding row sees nothing
    if (A.plan.n_split == 1)
      for (int i = tid; i < nh * HD / 4; i += 64 * KV8_WAVES) {
        const float z[4] = {0.f, 0.f, 0.f, 0.f};
        put<OUT>(A, r, head0 + i / (HD / 4), i % (HD / 4) * 4, z);
      }
    return;
  }
  const int ctx = min(pos + 1, kv8_most(A.c, A.b));
  const int64_t c0l = (int64_t)split * A.plan.chunk;
  if (c0l >= ctx) return;
  const int c0 = (int)c0l, c1 = split == A.plan.n_split - 1 ? ctx : min(ctx, c0 + A.plan.chunk);
  const int steps = (c1 - c0 + 31) / 32, last_blk = (c1 - 1) >> 4;
  const int mine = (steps - wave + KV8_WAVES - 1) / KV8_WAVES;   // steps wave, wave + 4, ...
  const int32_t* tab = kv8_table(A.b, s);

  bf16x8_t qf[2 * NJ][QP];
  {
    const T* qp = (const T*)A.q.p + r * A.q.row + (head0 + col) * A.q.head;
    const bool vec = (((uintptr_t)A.q.p | (A.q.row * sizeof(T)) | (A.q.head * sizeof(T))) & 15) == 0;
#pragma unroll
    for (int kk = 0; kk < 2 * NJ; ++kk)
      query8<T, QP>(qp + 64 * (kk >> 1) + 16 * grp + 8 * (kk & 1), col < nh, vec, qf[kk]);
  }
  const float sc = A.scale * KV8_LOG2E;
  float m = -INFINITY, l = 0.f;
  f32x4_t o[NJ][4];
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[j][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  const uint8_t* kl = A.c.k + lane * 16;
  const uint8_t* vl = A.c.v + grp * (4 * HD) + col * 16;
  u32x4_t kr[2][NJ], vr[2][NJ];
  int ids = 0;                      // lane i: block i & 1 of step i >> 1 of the current 32 steps
  float kss = 1.f, vss = 1.f;
  auto lists = [&](int i0) {
    const int st = wave + KV8_WAVES * (i0 + (lane >> 1));
    const int blk = min((c0 >> 4) + 2 * st + (lane & 1), last_blk);
    ids = kv8_block(A.c, tab, A.b.tab_stride, blk, kvh);
    kss = ids < 0 ? 1.f : A.c.k_scale[ids];
    vss = ids < 0 ? 1.f : A.c.v_scale[ids];
  };
  auto fetch = [&](int i) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int id = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + h);
      if (id < 0) {                 // a page the pool has not: its tokens are NaN
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          kr[h][j] = u32x4_t{KV8_NAN4, KV8_NAN4, KV8_NAN4, KV8_NAN4};
          vr[h][j] = u32x4_t{0, 0, 0, 0};
        }
      } else {
        const int64_t at = (int64_t)id * (16 * HD);
#pragma unroll
        for (int j = 0; j < NJ; ++j) kr[h][j] = *reinterpret_cast<const u32x4_t*>(kl + at + j * 1024);
#pragma unroll
        for (int j = 0; j < NJ; ++j) vr[h][j] = *reinterpret_cast<const u32x4_t*>(vl + at + j * 256);
      }
    }
  };
  if (mine > 0) {
    lists(0);
    fetch(0);
  }
  for (int i = 0; i < mine; ++i) {
    const int t0 = c0 + 32 * (wave + KV8_WAVES * i);
    float ks[2], vs[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ks[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(kss), 2 * (i & 31) + h));
      vs[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vss), 2 * (i & 31) + h));
    }
    u32x4_t kc[2][NJ], vc[2][NJ];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        kc[h][j] = kr[h][j];
        vc[h][j] = vr[h][j];
      }
    if (i + 1 < mine) {             // the next step's loads run under this step's products
      if (((i + 1) & 31) == 0) lists(i + 1);
      fetch(i + 1);
    }
    f32x4_t st[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      st[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bf16x8_t kf = kv8_bf16x8(kc[h][j][2 * e], kc[h][j][2 * e + 1], ks[h], ks[h]);
#pragma unroll
          for (int n = 0; n < QP; ++n)
            st[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[2 * j + e][n], st[h], 0, 0, 0);
        }
    }
    // lane's tokens: 16 h + 4 grp + e of the step
    const int left = c1 - t0;       // tokens of the step that the chunk has
    if (left < 32) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * h + 4 * grp + e >= left) st[h][e] = -INFINITY;
        // stale slots may hold NaN codes, and 0 * NaN is NaN: clear them
        const int n = min(max(left - 16 * h - 4 * grp, 0), 4);
        const uint32_t keep = n == 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u;
#pragma unroll
        for (int j = 0; j < NJ; ++j) vc[h][j] &= keep;
      }
    }
    float mx = fmaxf(fmaxf(fmaxf(st[0][0], st[0][1]), fmaxf(st[0][2], st[0][3])),
                     fmaxf(fmaxf(st[1][0], st[1][1]), fmaxf(st[1][2], st[1][3]))) * sc;
    if (i == 0 || __any(mx > m + KV8_SLACK)) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = fmaxf(m, mx);
      const float alpha = i == 0 ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      l *= alpha;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] *= alpha;
      m = mn;
    }
    float p[8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[4 * h + e] = __builtin_amdgcn_exp2f(fmaf(st[h][e], sc, -m));
        l += p[4 * h + e];
      }
    bf16x8_t pf[PP];
    operand8<PP>(p, pf);
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bf16x8_t vf = kv8_bf16x8(vc[0][j][e], vc[1][j][e], vs[0], vs[1]);
#pragma unroll
        for (int n = 0; n < PP; ++n) o[j][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n], o[j][e], 0, 0, 0);
      }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  // join the waves: column `col`, dims 64 j + 16 grp + 4 i + e of the lane
  if (col < nh) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4_t*>(&sO[wave][col][64 * j + 16 * grp + 4 * i]) =
            f32x4_t{o[j][0][i], o[j][1][i], o[j][2][i], o[j][3][i]};
    if (grp == 0) {
      sM[wave][col] = m;
      sL[wave][col] = l;
    }
  }
  __syncthreads();
  const int64_t slot = (int64_t)r * A.plan.n_split + split;
  for (int i = tid; i < nh * (HD / 4); i += 64 * KV8_WAVES) {
    const int h = i / (HD / 4), d = i % (HD / 4) * 4;
    const int nw = min(steps, KV8_WAVES);        // waves that had a step
    float M = sM[0][h];
    for (int w = 1; w < nw; ++w) M = fmaxf(M, sM[w][h]);
    float L = 0.f;
    f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < nw; ++w) {
      const float f = __builtin_amdgcn_exp2f(sM[w][h] - M);
      L += f * sL[w][h];
      acc += f * *reinterpret_cast<const f32x4_t*>(&sO[w][h][d]);
    }
    if (A.plan.n_split == 1) {
      const float inv = 1.0f / L;
      const float v[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
      put<OUT>(A, r, head0 + h, d, v);
    } else {
      const float v[4] = {acc[0], acc[1], acc[2], acc[3]};
      put_part(A, slot, head0 + h, d, v);
      if (d == 0) {
        float* ml = part_ml(A, slot, head0 + h);
        ml[0] = M;
        ml[1] = L;
      }
    }
  }
}

// ---------------------------------------------------------------- tiles pass
__device__ __forceinline__ bool has_nan_code(uint32_t w) { return (((w & KV8_NAN4) + 0x01010101u) & 0x80808080u) != 0; }

// Four codes with NaN ones cleared.
__device__ __forceinline__ uint32_t clear_nan(uint32_t w) {
  const uint32_t hit = (((w & KV8_NAN4) + 0x01010101u) & 0x80808080u) >> 7;
  return w & ~(hit * 0xFFu);
}

template <typename T, int HD, int OUT>
__global__ __launch_bounds__(64 * KV8_WAVES, 2) void k_kv8_tiles(Kv8Attn A, int tiles) {
  constexpr int QP = q_pieces(OUT), PP = p_pieces(OUT, true);
  constexpr int NK = HD / 16;       // 32x32x16 steps over the head's dims
  constexpr int DT = HD / 32;       // 32-dim tiles of the output: tile e holds dims DT * row + e
  constexpr int BLK = 16 * HD;      // bytes of a block
  constexpr int PASSES = 4 * BLK / (256 * 16);   // 16-byte loads per thread and operand
  __shared__ __attribute__((aligned(16))) uint8_t sK[2][4 * BLK], sV[2][4 * BLK];
  __shared__ float sS[2][8];        // key, then value scales of the four blocks

  // Blocks are dealt to the 8 XCDs in turn, so with the kv heads side by side an
  // XCD keeps to few of them.  Tiles go last first: within a sequence the
  // longest contexts start first.
  int64_t item = blockIdx.x;
  const int kvh = (int)(item % A.c.n_kv);
  item /= A.c.n_kv;
  const int split = (int)(item % A.plan.n_split);
  const int k = tiles - 1 - (int)(item / A.plan.n_split);
  const int rep = A.n_q / A.c.n_kv, np = KV8_TILE_Q / rep;
  int key, s, r0, n;
  s = kv8_find(A.b, k, np, 1, key);
  kv8_seq_rows(A.b, s, r0, n);
  const int skip = (k - key) * np;  // rows of the sequence before the tile
  const int nr = min(np, n - skip);
  if (nr <= 0) return;
  const int pos0 = A.b.seq_len[s] + A.b.len_add - n + skip;   // position of the tile's first row
  r0 += skip;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c32 = lane & 31, hh = lane >> 5;
  const int qi = wave * 32 + c32;
  const bool valid = qi < nr * rep;
  const int row = r0 + (valid ? qi / rep : 0), head = kvh * rep + (valid ? qi % rep : 0);
  const int most = kv8_most(A.c, A.b);
  const int limit = valid ? min(pos0 + qi / rep + 1, most) : 0;      // tokens the column sees
  const int wmax = pos0 + min(nr - 1, (wave * 32 + 31) / rep) + 1;   // most of any column of the wave
  const bool active = wave * 32 < nr * rep;
  const int end = min(pos0 + nr, most);   // tokens that the tile's last row sees
  const int64_t c0l = (int64_t)split * A.plan.chunk;
  if (A.plan.n_split > 1 && c0l >= end) return;
  const int c0 = (int)c0l, c1 = split == A.plan.n_split - 1 ? end : min(end, c0 + A.plan.chunk);
  const int32_t* tab = kv8_table(A.b, s);

  bf16x8_t qf[NK][QP];
  {
    const T* qp = (const T*)A.q.p + row * A.q.row + head * A.q.head;
    const bool vec = (((uintptr_t)A.q.p | (A.q.row * sizeof(T)) | (A.q.head * sizeof(T))) & 15) == 0;
#pragma unroll
    for (int kk = 0; kk < NK; ++kk)
      query8<T, QP>(qp + 16 * (2 * (kk >> 1) + hh) + 8 * (kk & 1), valid, vec, qf[kk]);
  }
  const float sc = A.scale * KV8_LOG2E;
  float m = -INFINITY, l = 0.f;
  f32x16_t o[DT];
#pragma unroll
  for (int e = 0; e < DT; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[e][i] = 0.f;

  // A pass of the workgroup's 16-byte loads covers whole blocks by whole waves:
  // a wave's block ids and scales are scalars.
  const int last_blk = (max(c1, 1) - 1) >> 4;
  u32x4_t kr[PASSES], vr[PASSES];
  float ksr[PASSES], vsr[PASSES];
  int ids[PASSES];
  auto piece = [&](int p) { return (p * 256 + wave * 64) * 16 / BLK; };   // block of the wave's piece in pass p
  auto list = [&](int t0) {
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
      ids[p] = __builtin_amdgcn_readfirstlane(
          kv8_block(A.c, tab, A.b.tab_stride, min((t0 >> 4) + piece(p), last_blk), kvh));
  };
  auto fetch = [&]() {
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int off = (p * 256 + tid) * 16 % BLK;
      if (ids[p] < 0) {             // a page the pool has not: its tokens are NaN
        kr[p] = u32x4_t{KV8_NAN4, KV8_NAN4, KV8_NAN4, KV8_NAN4};
        vr[p] = u32x4_t{0, 0, 0, 0};
        ksr[p] = vsr[p] = 1.f;
      } else {
        kr[p] = *reinterpret_cast<const u32x4_t*>(A.c.k + (int64_t)ids[p] * BLK + off);
        vr[p] = *reinterpret_cast<const u32x4_t*>(A.c.v + (int64_t)ids[p] * BLK + off);
        ksr[p] = A.c.k_scale[ids[p]];
        vsr[p] = A.c.v_scale[ids[p]];
      }
    }
  };
  auto stash = [&](int buf) {
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      *reinterpret_cast<u32x4_t*>(&sK[buf][(p * 256 + tid) * 16]) = kr[p];
      *reinterpret_cast<u32x4_t*>(&sV[buf][(p * 256 + tid) * 16]) = vr[p];
      if (lane == 0) {
        sS[buf][piece(p)] = ksr[p];
        sS[buf][4 + piece(p)] = vsr[p];
      }
    }
  };
  auto block = [&](int buf, int t0) {
    f32x16_t st[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int i = 0; i < 16; ++i) st[u][i] = 0.f;
      const int b = 2 * u + (c32 >> 4);
      const float ks = sS[buf][b];
      const uint8_t* kp = &sK[buf][b * BLK + (c32 & 15) * 16 + hh * 256];
#pragma unroll
      for (int j = 0; j < NK / 2; ++j) {
        const u32x4_t w = *reinterpret_cast<const u32x4_t*>(kp + j * 512);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bf16x8_t kf = kv8_bf16x8(w[2 * e], w[2 * e + 1], ks, ks);
#pragma unroll
          for (int n = 0; n < QP; ++n)
            st[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[2 * j + e][n], st[u], 0, 0, 0);
        }
      }
    }
    // lane's tokens: 32 u + 8 (i / 4) + 4 hh + i % 4
    const bool masked = __any(valid && t0 + 64 > limit);
    if (masked) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (t0 + 32 * u + 8 * (i / 4) + 4 * hh + i % 4 >= limit) st[u][i] = -INFINITY;
    }
    float mx = st[0][0];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[u][i]);
    mx *= sc;
    if (__any(mx > m + KV8_SLACK)) {
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = fmaxf(m, mx);
      const float alpha = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);   // -inf: nothing seen yet
      l *= alpha;
#pragma unroll
      for (int e = 0; e < DT; ++e) o[e] *= alpha;
      m = mn;
    }
    // a column that sees none of the tokens so far keeps m = -inf: its
    // probabilities are exp2(-inf) = 0
    const float ms = m == -INFINITY ? 0.f : m;
    bf16x8_t pf[4][PP];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(st[u][8 * a + e], sc, -ms));
          l += p[e];
        }
        operand8<PP>(p, pf[2 * u + a]);
      }
    bool nan = false;
#pragma unroll
    for (int b = 0; b < 4; ++b) {   // 16 tokens: value rows 4 hh .. + 3 and 8 + 4 hh .. + 3
      const uint8_t* vp = &sV[buf][b * BLK + hh * (4 * HD) + c32 * (4 * DT)];
      uint32_t lo[DT], hi[DT];
      if constexpr (DT == 4) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(vp), y = *reinterpret_cast<const u32x4_t*>(vp + 8 * HD);
#pragma unroll
        for (int e = 0; e < 4; ++e) { lo[e] = x[e]; hi[e] = y[e]; }
      } else {
        const u32x2_t x = *reinterpret_cast<const u32x2_t*>(vp), y = *reinterpret_cast<const u32x2_t*>(vp + 8 * HD);
#pragma unroll
        for (int e = 0; e < 2; ++e) { lo[e] = x[e]; hi[e] = y[e]; }
      }
      if (masked) {                 // 0 * NaN is NaN: masked tokens' NaN codes must not reach the product
#pragma unroll
        for (int e = 0; e < DT; ++e) {
          nan |= has_nan_code(lo[e]) | has_nan_code(hi[e]);
          lo[e] = clear_nan(lo[e]);
          hi[e] = clear_nan(hi[e]);
        }
      }
      const float vs = sS[buf][4 + b];
#pragma unroll
      for (int e = 0; e < DT; ++e) {
        const bf16x8_t vf = kv8_bf16x8(lo[e], hi[e], vs, vs);
#pragma unroll
        for (int n = 0; n < PP; ++n) o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[b][n], o[e], 0, 0, 0);
      }
    }
    if (__any(nan)) {               // NaN values: those a column does see make its dims NaN
      for (int t = 0; t < 64; ++t) {
        if (t0 + t >= limit) break;
        const uint8_t* vp = &sV[buf][(t >> 4) * BLK + ((t >> 2) & 3) * (4 * HD) + (t & 3)];
#pragma unroll
        for (int e = 0; e < DT; ++e)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if ((vp[(DT * (8 * (i / 4) + 4 * hh + i % 4) + e) * 4] & 0x7F) == 0x7F) o[e][i] = __uint_as_float(0x7FC00000u);
      }
    }
  };

  if (c0 < c1) {
    list(c0);
    fetch();
    list(c0 + 64);
    int buf = 0;
    for (int t0 = c0; t0 < c1; t0 += 64, buf ^= 1) {
      stash(buf);
      __syncthreads();              // the piece is in LDS; the other buffer is free
      if (t0 + 64 < c1) {
        fetch();
        list(t0 + 128);
      }
      if (active && t0 < wmax) block(buf, t0);
    }
  }
  if (!active) return;
  l += __shfl_xor(l, 32, 64);
  if (!valid) return;
  // a lane's outputs: dims DT * (8 (i / 4) + 4 hh + i % 4) + e
  constexpr int NV = 4 * DT;        // consecutive dims for one i / 4
  if (A.plan.n_split == 1) {
    const float inv = limit > 0 ? 1.0f / l : 0.f;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float v[NV];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < DT; ++e) v[DT * i + e] = o[e][4 * g + i] * inv;
      put<OUT>(A, row, head, DT * (8 * g + 4 * hh), v);
    }
  } else if (limit > c0) {
    const int64_t slot = (int64_t)row * A.plan.n_split + split;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float v[NV];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < DT; ++e) v[DT * i + e] = o[e][4 * g + i];
      put_part(A, slot, head, DT * (8 * g + 4 * hh), v);
    }
    if (hh == 0) {
      float* ml = part_ml(A, slot, head);
      ml[0] = m;
      ml[1] = l;
    }
  }
}

// ---------------------------------------------------------------- merge
// One workgroup per (row, head): a wave takes every fourth chunk, a lane HD / 64 dims.
template <int HD, int OUT>
__global__ __launch_bounds__(256) void k_kv8_merge(Kv8Attn A) {
  constexpr int NV = HD / 64;
  __shared__ float sO[4][HD], sM[4], sL[4];
  const int r = blockIdx.x, h = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int s, pos;
  if (!kv8_row(A.b, r, s, pos)) return;
  const int ctx = min(pos + 1, kv8_most(A.c, A.b));
  const int n = ctx <= 0 ? 0 : min((ctx - 1) / A.plan.chunk + 1, A.plan.n_split);
  float m = -INFINITY, l = 0.f, o[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) o[i] = 0.f;
  for (int c = wave; c < n; c += 4) {
    const int64_t slot = (int64_t)r * A.plan.n_split + c;
    const float* ml = part_ml(A, slot, h);
    const float* po = A.part_o + (slot * A.n_q + h) * HD + lane * NV;
    float v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = po[i];
    const float mc = ml[0], lc = ml[1], mn = fmaxf(m, mc);
    const float a = c == wave ? 0.f : __builtin_amdgcn_exp2f(m - mn), f = __builtin_amdgcn_exp2f(mc - mn);
    l = l * a + lc * f;
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] = o[i] * a + v[i] * f;
    m = mn;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) sO[wave][lane * NV + i] = o[i];
  if (lane == 0) {
    sM[wave] = m;
    sL[wave] = l;
  }
  __syncthreads();
  if (tid >= HD / 4) return;
  const int d = tid * 4, nw = min(n, 4);
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (nw > 0) {
    float M = sM[0];
    for (int w = 1; w < nw; ++w) M = fmaxf(M, sM[w]);
    float L = 0.f;
    for (int w = 0; w < nw; ++w) {
      const float f = __builtin_amdgcn_exp2f(sM[w] - M);
      L += f * sL[w];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += f * sO[w][d + i];
    }
    const float inv = 1.0f / L;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] *= inv;
  }
  put<OUT>(A, r, h, d, v);
}

template <typename F, typename... Args>
void launch(F kernel, dim3 grid, dim3 block, hipStream_t st, Args... args) {
  hipEvent_t e0, e1;
  if (rg_take_launch_events(&e0, &e1))
    hipExtLaunchKernelGGL(kernel, grid, block, 0, st, e0, e1, 0, args...);
  else
    hipLaunchKernelGGL(kernel, grid, block, 0, st, args...);
}

template <typename T, int HD, int OUT>
hipError_t run(const Kv8Attn& a, hipStream_t st) {
  const int rep = a.n_q / a.c.n_kv;
  if (a.plan.tiles) {
    const int np = KV8_TILE_Q / rep;
    const int64_t tiles = (int64_t)a.b.rows / np + a.b.n_seqs, grid = tiles * a.c.n_kv * a.plan.n_split;
    if (grid > INT32_MAX) return hipErrorInvalidValue;
    launch(k_kv8_tiles<T, HD, OUT>, dim3((unsigned)grid), dim3(64 * KV8_WAVES), st, a, (int)tiles);
  } else {
    const int htiles = (rep + 15) / 16;
    const int64_t items = (int64_t)a.b.rows * a.c.n_kv * htiles * a.plan.n_split, per = (items + 7) / 8;
    if (8 * per > INT32_MAX) return hipErrorInvalidValue;
    launch(k_kv8_rows<T, HD, OUT>, dim3((unsigned)(8 * per)), dim3(64 * KV8_WAVES), st, a, htiles, (int)per, items);
  }
  return hipGetLastError();
}

template <int HD, int OUT>
hipError_t merge(const Kv8Attn& a, hipStream_t st) {
  launch(k_kv8_merge<HD, OUT>, dim3(a.b.rows, a.n_q), dim3(256), st, a);
  return hipGetLastError();
}

}  // namespace

// Rows or tiles: a tile's 128 query rows pay from a few rows a sequence on; below,
// the rows pass keeps the matrix units no busier than the memory.  Chunks: as
// many as give the chip about four workgroups a CU, of at least 512 tokens.
Kv8Plan kv8_plan(int rows, int n_seqs, bool has_off, int n_q, int n_kv, int max_len, int max_split) {
  Kv8Plan p{};
  const int rep = n_q / n_kv;
  p.tiles = has_off && rep <= KV8_TILE_Q && (int64_t)rows >= 4LL * n_seqs;
  const int64_t wgs = p.tiles ? ((int64_t)rows * rep + KV8_TILE_Q - 1) / KV8_TILE_Q * n_kv
                              : (int64_t)rows * n_kv * ((rep + 15) / 16);
  int64_t n = std::min<int64_t>((1024 + wgs - 1) / wgs, (max_len + 511) / 512);
  n = std::max<int64_t>(1, std::min<int64_t>(n, max_split));
  p.chunk = (int)std::min<int64_t>((((int64_t)max_len + n - 1) / n + 63) / 64 * 64, 1 << 30);
  p.n_split = (int)((max_len + (int64_t)p.chunk - 1) / p.chunk);
  if (p.n_split < 1) p.n_split = 1;
  return p;
}

hipError_t launch_kv8_attention(int dtype, bool planes, const Kv8Attn& a, hipStream_t st) {
  if (a.b.rows <= 0 || a.b.n_seqs <= 0) return hipSuccess;
  if ((a.c.hd != 64 && a.c.hd != 128) || a.plan.n_split < 1 || a.plan.chunk % 64 || (a.plan.n_split > 1 && (!a.part_o || !a.part_ml)))
    return hipErrorInvalidValue;
  const bool w = a.c.hd == 128;
  if (planes && dtype != 0) return hipErrorInvalidValue;
  if (planes) return w ? run<float, 128, OUT_PLANES>(a, st) : run<float, 64, OUT_PLANES>(a, st);
  if (dtype == 1) return w ? run<bf16_t, 128, OUT_BF16>(a, st) : run<bf16_t, 64, OUT_BF16>(a, st);
  return w ? run<float, 128, OUT_F32>(a, st) : run<float, 64, OUT_F32>(a, st);
}

hipError_t launch_kv8_merge(int dtype, bool planes, const Kv8Attn& a, hipStream_t st) {
  if (a.b.rows <= 0 || a.b.n_seqs <= 0 || a.plan.n_split <= 1) return hipSuccess;
  const bool w = a.c.hd == 128;
  if (planes) return w ? merge<128, OUT_PLANES>(a, st) : merge<64, OUT_PLANES>(a, st);
  if (dtype == 1) return w ? merge<128, OUT_BF16>(a, st) : merge<64, OUT_BF16>(a, st);
  return w ? merge<128, OUT_F32>(a, st) : merge<64, OUT_F32>(a, st);
}
