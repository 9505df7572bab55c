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
//   Its four or eight waves take 32-token steps in turn straight from memory, 16
//   bytes a lane, and join in LDS.  Bound by the cache's bytes: three rows of 60 to
//   131 thousand tokens, 4 kv heads (221 MB) 38 us, 5.9 TB/s of the 6.6 that a plain
//   read reaches; 512 rows of 512 to 2600 tokens, 2 kv heads 57 us.
// * Tiles pass (runs of rows): a workgroup per 128 query rows (positions x heads
//   of a kv head) and chunk.  32-token pieces go through LDS once for the four
//   waves of 32 query rows.  Bound by vector issue beside the matrix instructions:
//   8192 bf16 rows of 28 heads behind 2 to 6 thousand tokens (0.61 Tflop) 630 us,
//   0.97 of the 1.42 Pflop/s that a large product reaches.
// * With several chunks a row, a merge joins their partial results in order.
#include <algorithm>
#include <type_traits>

#include "kv8_attn_device.h"

namespace {

constexpr int KV8_TILE_Q = 128;     // query rows of a tile
constexpr int KV8_WAVES = 4;

enum { OUT_F32 = 0, OUT_BF16 = 1, OUT_PLANES = 2 };

// bf16 pieces of a query, and of a probability in either pass.
constexpr int q_pieces(int out) { return out == OUT_F32 ? 3 : out == OUT_PLANES ? 2 : 1; }
constexpr int p_pieces(int out, bool tiles) { return out == OUT_F32 ? 3 : out == OUT_PLANES || !tiles ? 2 : 1; }

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
// Work by length.  An XCD takes an eighth of the rows, in segments of 64, each from
// its longest row down; every other round of 32 blocks, one for each of its CUs,
// runs backwards, so that the CUs' sums even out.  512 rows of 512 to 2600 tokens
// and 2 kv heads: 60 us in place of 68 (47 where all have the same length); over
// all XCDs instead of within one 69, since siblings then share no L2.  Rows that are
// equal pay for it: 66 us in place of 64.
//
// The row of this block of an XCD, its kv head and head tile, tokens and table row;
// false where there is none.  The row of a rank is found bit by bit of the lengths
// in 32-token steps, a row a lane.
__device__ __forceinline__ bool deal_item(const Kv8Attn& A, int htiles, int& r, int& kvh, int& ht, int& tokens, int& tab_row) {
  const int n = A.b.d_rows ? min(*A.b.d_rows, A.b.rows) : A.b.rows, per = (n + 7) >> 3, xcd = blockIdx.x & 7;
  const unsigned inner = (unsigned)(A.c.n_kv * htiles), span = 64 * inner;
  unsigned j = blockIdx.x >> 3;
  int row0 = xcd * per;
  if (j >= span) {
    const unsigned seg = j / span;
    row0 += 64 * (int)seg;
    j -= seg * span;
  }
  const int here = min(64, min(per * (xcd + 1), n) - row0);
  if (here <= 0) return false;
  const unsigned count = (unsigned)here * inner;
  if (j >= count) return false;
  const int lane = threadIdx.x & 63, bits = A.plan.deal;
  int len = 0, tr = row0 + lane;
  if (lane < here) {
    len = kv8_len(A.b, row0 + lane);
    if (A.b.tab_row) tr = A.b.tab_row[row0 + lane];
  }
  const unsigned p = (j & 32) && (j | 31) < count ? (j & ~31u) + 31 - (j & 31) : j, rank = p / inner, rest = p - rank * inner;
  const int key = min((int)(((unsigned)len + 31) >> 5), (1 << bits) - 1);
  uint64_t left = here == 64 ? ~0ull : (1ull << here) - 1;
  int k = (int)rank;
  for (int bit = bits - 1; bit >= 0; --bit) {
    const uint64_t set = __ballot(key >> bit & 1) & left;
    const int c = __popcll(set);
    left = k < c ? set : left & ~set;
    k -= k < c ? 0 : c;
  }
  const int at = wave_nth_bit(left, k);
  r = row0 + at;
  ht = htiles == 1 ? 0 : (int)(rest / (unsigned)A.c.n_kv);
  kvh = (int)rest - ht * A.c.n_kv;
  tokens = __builtin_amdgcn_readlane(len, at);
  tab_row = __builtin_amdgcn_readlane(tr, at);
  return true;
}

template <typename T, int HD, int OUT, int W>
__global__ __launch_bounds__(64 * W, (sizeof(T) == 2 || HD == 64 ? 4 : 3) * 4 / W) void k_kv8_rows(
    Kv8Attn A, int htiles, int per_xcd, int items) {
  constexpr int QP = q_pieces(OUT), PP = p_pieces(OUT, false);
  constexpr int NJ = HD / 64;       // 16-byte loads of a block per lane
  constexpr int LDO = HD + 4;
  __shared__ __attribute__((aligned(16))) float sO[W][16][LDO];
  __shared__ float sM[W][16], sL[W][16];

  // Blocks are dealt to the 8 XCDs in turn: neighbouring rows, which share
  // pages where they are siblings of a prompt, go to the same one.
  int r, kvh, ht, split = 0, pos;
  const int32_t* tab;
  if (A.plan.deal) {
    int tokens, tr;
    if (!deal_item(A, htiles, r, kvh, ht, tokens, tr)) return;
    pos = tokens - 1;
    tab = (unsigned)tr < (unsigned)A.b.tab_rows ? A.b.tab + (int64_t)tr * A.b.tab_stride : nullptr;
  } else {
    unsigned item = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (item >= (unsigned)items) return;
    split = (int)(item % (unsigned)A.plan.n_split);
    item /= (unsigned)A.plan.n_split;
    ht = (int)(item % (unsigned)htiles);
    item /= (unsigned)htiles;
    kvh = (int)(item % (unsigned)A.c.n_kv);
    r = (int)(item / (unsigned)A.c.n_kv);
    int s;
    if (!kv8_row(A.b, r, s, pos)) return;
    tab = kv8_table(A.b, s);
  }
  const int rep = A.n_q / A.c.n_kv, nh = min(16, rep - ht * 16), head0 = kvh * rep + ht * 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  if (pos < 0) {                    // a padding row sees nothing
    if (A.plan.n_split == 1)
      for (int i = tid; i < nh * HD / 4; i += 64 * W) {
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
  const int mine = (steps - wave + W - 1) / W;   // steps wave, wave + W, ...

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
    const int st = wave + W * (i0 + (lane >> 1));
    const int blk = min((c0 >> 4) + 2 * st + (lane & 1), last_blk);
    ids = kv8_block(A.c, tab, A.b.tab_stride, blk, kvh);
    kss = ids < 0 ? 1.f : A.c.k_scale[ids];
    vss = ids < 0 ? 1.f : A.c.v_scale[ids];
  };
  auto fetch_k = [&](int i) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* p = kl + (int64_t)max(__builtin_amdgcn_readlane(ids, 2 * (i & 31) + h), 0) * (16 * HD);
#pragma unroll
      for (int j = 0; j < NJ; ++j) kr[h][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p + j * 1024));
    }
  };
  auto fetch_v = [&](int i) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* p = vl + (int64_t)max(__builtin_amdgcn_readlane(ids, 2 * (i & 31) + h), 0) * (16 * HD);
#pragma unroll
      for (int j = 0; j < NJ; ++j) vr[h][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p + j * 256));
    }
  };
  // The first step's keys, the queries, the values: all on their way before the
  // first of them is waited for (queries first, and waited for: 59 us in place of 57).
  constexpr int NW = sizeof(T) / 2;
  const T* qp = (const T*)A.q.p + r * A.q.row + (head0 + col) * A.q.head;
  const bool vec = (((uintptr_t)A.q.p | (A.q.row * sizeof(T)) | (A.q.head * sizeof(T))) & 15) == 0;
  u32x4_t raw[2 * NJ][NW];
  if (mine > 0) {
    lists(0);
    fetch_k(0);
  }
#pragma unroll
  for (int kk = 0; kk < 2 * NJ; ++kk)
#pragma unroll
    for (int w = 0; w < NW; ++w)
      raw[kk][w] = vec && col < nh ? *reinterpret_cast<const u32x4_t*>(qp + 64 * (kk >> 1) + 16 * grp + 8 * (kk & 1) + w * (16 / sizeof(T)))
                                   : u32x4_t{0, 0, 0, 0};
  if (mine > 0) fetch_v(0);
  bf16x8_t qf[2 * NJ][QP];
#pragma unroll
  for (int kk = 0; kk < 2 * NJ; ++kk) {
    if (!vec) {
      query8<T, QP>(qp + 64 * (kk >> 1) + 16 * grp + 8 * (kk & 1), col < nh, false, qf[kk]);
    } else if constexpr (sizeof(T) == 2) {
      qf[kk][0] = __builtin_bit_cast(bf16x8_t, raw[kk][0]);
    } else {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(raw[kk][e / 4][e & 3]);
      operand8<QP, QP == 3>(v, qf[kk]);
    }
  }
  for (int i = 0; i < mine; ++i) {
    const int t0 = c0 + 32 * (wave + W * i);
    float ks[2], vs[2];
    int lost = 0;                   // negative: a page the pool has not
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int id = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + h);
      lost |= id;
      ks[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(kss), 2 * (i & 31) + h));
      vs[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vss), 2 * (i & 31) + h));
    }
    // a lost page's tokens: NaN scores (the codes in the registers are another page's)
    const float none = lost < 0 ? __uint_as_float(0x7FC00000u) : 0.f;
    f32x4_t st[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      st[h] = f32x4_t{none, none, none, none};
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bf16x8_t kf = kv8_bf16x8(kr[h][j][2 * e], kr[h][j][2 * e + 1], ks[h], ks[h]);
#pragma unroll
          for (int n = 0; n < QP; ++n)
            st[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[2 * j + e][n], st[h], 0, 0, 0);
        }
    }
    // the next step's keys into the registers just read: they arrive under the
    // softmax and the values' products, and other waves' work
    if (i + 1 < mine) {
      if (((i + 1) & 31) == 0) lists(i + 1);
      fetch_k(i + 1);
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
        for (int j = 0; j < NJ; ++j) vr[h][j] &= keep;
      }
    }
    float mx = fmaxf(fmaxf(fmaxf(st[0][0], st[0][1]), fmaxf(st[0][2], st[0][3])),
                     fmaxf(fmaxf(st[1][0], st[1][1]), fmaxf(st[1][2], st[1][3]))) * sc;
    if (__any(mx > m + KV8_SLACK)) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = fmaxf(m, mx);
      const float alpha = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);   // -inf: only scores past fp32's range so far
      l *= alpha;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] *= alpha;
      m = mn;
    }
    const float ms = m == -INFINITY ? 0.f : m;   // then every score is -inf and its probability 0
    float p[8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[4 * h + e] = __builtin_amdgcn_exp2f(fmaf(st[h][e], sc, -ms));
        l += p[4 * h + e];
      }
    bf16x8_t pf[PP];
    operand8<PP>(p, pf);
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bf16x8_t vf = kv8_bf16x8(vr[0][j][e], vr[1][j][e], vs[0], vs[1]);
#pragma unroll
        for (int n = 0; n < PP; ++n) o[j][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n], o[j][e], 0, 0, 0);
      }
    if (i + 1 < mine) fetch_v(i + 1);
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
  for (int i = tid; i < nh * (HD / 4); i += 64 * W) {
    const int h = i / (HD / 4), d = i % (HD / 4) * 4;
    const int nw = min(steps, W);        // waves that had a step
    float M = sM[0][h];
    for (int w = 1; w < nw; ++w) M = fmaxf(M, sM[w][h]);
    float L = 0.f;
    f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < nw; ++w) {
      const float f = sM[w][h] == M ? 1.f : __builtin_amdgcn_exp2f(sM[w][h] - M);
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
// Tile k of a batch, tiles of np rows: among 64 sequences, a lane each, those with
// the longest contexts come first, so that none of them starts when the others end:
// 24 fp32 runs of 37 to 701 rows 78 us, 87 with each sequence's tiles in turn; bf16
// 40 and 46.  Equal ones pay for it: four of 2048 rows 651 us in place of 643.
// A sequence of T tiles behind `old` tokens has them at levels old / np + 1 .. old /
// np + T; level and place of a rank are found bit by bit.  False past the last tile.
__device__ __forceinline__ bool tile_of(const Kv8Rows& b, int np, int k, int& s, int& r0, int& n, int& skip) {
  auto key = [&](int q) { return min(max(b.seq_off[q], 0), b.rows) / np + q; };   // tiles are numbered from here
  int s0 = 0;
  for (int hi = (b.n_seqs + 63) >> 6, lo = 0; hi - lo > 1;) {
    const int mid = (lo + hi) >> 1;
    if (key(64 * mid) <= k) lo = mid;
    else hi = mid;
    s0 = 64 * lo;
  }
  const int lane = threadIdx.x & 63, rank = k - key(s0);
  int f = 0, c = 0, tiles = 0, top = 0;
  if (s0 + lane < b.n_seqs) {
    kv8_seq_rows(b, s0 + lane, f, c);
    tiles = (int)(((unsigned)max(c, 0) + np - 1) / (unsigned)np);
    top = (int)((unsigned)min(max(kv8_len(b, s0 + lane) - c, 0), 1 << 30) / (unsigned)np) + tiles;
  }
  auto from = [&](int level) { return wave_sum_dpp(min(max(top - level + 1, 0), tiles)); };   // tiles at it and above
  int level = 0;
  for (int bit = 31 - __clz(wave_max_dpp(top) | 1); bit >= 0; --bit)
    if (from(level | 1 << bit) > rank) level |= 1 << bit;
  if (rank < 0 || level == 0) return false;
  const int down = top - level;
  const int at = wave_nth_bit(__ballot(down >= 0 && down < tiles), rank - from(level + 1));
  s = s0 + at;
  r0 = __builtin_amdgcn_readlane(f, at);
  n = __builtin_amdgcn_readlane(c, at);
  skip = __builtin_amdgcn_readlane(tiles - 1 - down, at) * np;
  return true;
}

// Codes are converted once a workgroup, on their way into LDS: a wave that
// converted its own operands spent 128 of its 300 vector instructions per 64
// tokens on it.  A wave's chain through a piece (scores, maximum, exponentials,
// values) is several times longer than its matrix instructions take, so what
// counts is how many waves a SIMD has: pieces of 32 tokens and 168 registers leave
// room for three workgroups a CU.
//
// LDS, in 16-byte pieces.  Keys [dim / 8][token]: a piece is 8 dims of a token.
// Values [block][half hh][e][m]: a piece is dim DT m + e, tokens 4 hh .. + 3 and
// 8 + 4 hh .. + 3 of a block, those whose probabilities lane half hh holds.  Lanes
// read neighbouring pieces.
template <typename T, int HD, int OUT>
__global__ __launch_bounds__(64 * KV8_WAVES, OUT == OUT_BF16 ? 3 : 2) void k_kv8_tiles(Kv8Attn A) {
  constexpr int QP = q_pieces(OUT), PP = p_pieces(OUT, true);
  constexpr int NK = HD / 16;       // 32x32x16 steps over the head's dims
  constexpr int DT = HD / 32;       // 32-dim tiles of the output: tile e holds dims DT * row + e
  constexpr int BLK = 16 * HD;      // bytes of a block
  __shared__ u32x4_t sK[2][HD / 8][32], sV[2][2][2][DT][32];
  __shared__ int sNan[2][KV8_WAVES];

  // Blocks are dealt to the 8 XCDs in turn, so with the kv heads side by side an
  // XCD keeps to few of them.
  unsigned item = blockIdx.x;
  const int kvh = (int)(item % (unsigned)A.c.n_kv);
  item /= (unsigned)A.c.n_kv;
  const int split = (int)(item % (unsigned)A.plan.n_split);
  const int rep = A.n_q / A.c.n_kv, np = KV8_TILE_Q / rep;
  int s, r0, n, skip;               // the tile's sequence, its rows, those before the tile
  if (!tile_of(A.b, np, (int)(item / (unsigned)A.plan.n_split), s, r0, n, skip)) return;
  const int nr = min(np, n - skip);
  const int pos0 = kv8_len(A.b, s) - n + skip;   // position of the tile's first row
  r0 += skip;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c32 = lane & 31, hh = lane >> 5;
  const int qi = wave * 32 + c32;
  const bool valid = qi < nr * rep;
  const int row = r0 + (valid ? qi / rep : 0), head = kvh * rep + (valid ? qi % rep : 0);
  const int most = kv8_most(A.c, A.b);
  const int limit = valid ? min(pos0 + qi / rep + 1, most) : 0;      // tokens the column sees
  const int wmax = pos0 + min(nr - 1, (wave * 32 + 31) / rep) + 1;   // most of any column of the wave
  const int whole = min(pos0 + 1, most);  // tokens that every row of the tile sees
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
    for (int kk = 0; kk < NK; ++kk) query8<T, QP>(qp + 16 * kk + 8 * hh, valid, vec, qf[kk]);
  }
  const float sc = A.scale * KV8_LOG2E;
  float m = -INFINITY, l = 0.f;
  f32x16_t o[DT];
#pragma unroll
  for (int e = 0; e < DT; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[e][i] = 0.f;

  // Loads of a piece (2 blocks): 16 bytes of keys and 16 of values a thread (head
  // dim 128), or of one of them (64).  A wave's lie in one block, so its id and
  // scales are scalars.  What is loaded is first touched by the next stash: a
  // select on it here would wait for it.
  constexpr bool BOTH = HD == 128;
  const bool has_k = BOTH || wave < 2, has_v = BOTH || wave >= 2;
  const int wblk = BOTH ? wave >> 1 : wave & 1;
  const int piece = tid & (HD - 1);             // of the block
  const int last_blk = (max(c1, 1) - 1) >> 4;
  struct Load { u32x4_t k, v; float ks, vs; int id; };
  // Pieces in flight: two where two workgroups a CU leave the registers for it (fp32
  // runs 90 -> 86 us), one where a second set would spill (649 -> 730).
  constexpr int DEPTH = OUT == OUT_BF16 ? 1 : 2;
  Load ld[DEPTH];
  int id;
  auto list = [&](int t0) {
    id = __builtin_amdgcn_readfirstlane(kv8_block(A.c, tab, A.b.tab_stride, min((t0 >> 4) + wblk, last_blk), kvh));
  };
  auto fetch = [&](Load& x) {
    const int b = max(id, 0);
    const int64_t at = (int64_t)b * BLK + piece * 16;
    if (has_k) {
      x.k = *reinterpret_cast<const u32x4_t*>(A.c.k + at);
      x.ks = A.c.k_scale[b];
    }
    if (has_v) {
      x.v = *reinterpret_cast<const u32x4_t*>(A.c.v + at);
      x.vs = A.c.v_scale[b];
    }
    x.id = id;
  };
  auto stash = [&](Load& x, int buf, int t0) {
    if (x.id < 0) {                 // a page the pool has not: its keys are NaN, its values 0
      x.k = u32x4_t{KV8_NAN4, KV8_NAN4, KV8_NAN4, KV8_NAN4};
      x.v = u32x4_t{0, 0, 0, 0};
    }
    if (has_k) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        sK[buf][2 * (piece >> 4) + e][16 * wblk + (piece & 15)] =
            __builtin_bit_cast(u32x4_t, kv8_bf16x8(x.k[2 * e], x.k[2 * e + 1], x.ks, x.ks));
    }
    if (has_v) {
      if (t0 + 32 > whole) {        // some rows do not see all of these tokens: 0 * NaN must not reach them
        bool nan = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          nan |= has_nan_code(x.v[e]);
          x.v[e] = clear_nan(x.v[e]);
        }
        const bool any = __any(nan);
        if (lane == 0) sNan[buf][wave] = any;
      }
      const int tg = piece / (HD / 4), x4 = piece % (HD / 4);   // tokens 4 tg .., dims 4 x4 ..
      // a lost page's zeros do not take the scale of the block that was read in its place; in a scalar register,
      // as a vector one more costs bf16 rows 12 % (649 -> 730 us)
      const float vs = x.id < 0 ? 1.f : __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x.vs)));
#pragma unroll
      for (int d = 0; d < 4; ++d)
        reinterpret_cast<u32x2_t*>(&sV[buf][wblk][tg & 1][d % DT][(4 * x4 + d) / DT])[tg >> 1] = kv8_bf16x4(x.v[d], vs);
    }
  };
  // NaN values among the 32 tokens of a piece: those that a column does see make
  // its dims NaN.  A product counts them: ones at the NaN codes, ones at the tokens
  // in sight.
  auto nan_values = [&](int t0) {
#pragma unroll 1
    for (int b = 0; b < 2; ++b) {
      if (t0 + 16 * b >= c1) break;
      const int nid = kv8_block(A.c, tab, A.b.tab_stride, (t0 >> 4) + b, kvh);
      if (nid < 0) continue;        // its keys made the rows NaN
      const int left = limit - t0 - 16 * b - 4 * hh;
      uint32_t seen[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = i < 2 ? 2 * i : 4 + 2 * i;   // tokens t, t + 1 behind 4 hh
        seen[i] = (t < left ? 0x3F80u : 0u) | (t + 1 < left ? 0x3F800000u : 0u);
      }
      const uint32_t* vp = reinterpret_cast<const uint32_t*>(A.c.v + (int64_t)nid * BLK + hh * (4 * HD)) + DT * c32;
#pragma unroll
      for (int e = 0; e < DT; ++e) {
        uint32_t one[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t hit = (((vp[e + 2 * HD * h] & KV8_NAN4) + 0x01010101u) & 0x80808080u) >> 7;   // 1 in each such byte
          one[2 * h] = (hit & 1u) * 0x3F80u | (hit >> 8 & 1u) * 0x3F800000u;
          one[2 * h + 1] = (hit >> 16 & 1u) * 0x3F80u | (hit >> 24) * 0x3F800000u;
        }
        f32x16_t n;
#pragma unroll
        for (int i = 0; i < 16; ++i) n[i] = 0.f;
        n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8_t, u32x4_t{one[0], one[1], one[2], one[3]}),
            __builtin_bit_cast(bf16x8_t, u32x4_t{seen[0], seen[1], seen[2], seen[3]}), n, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (n[i] > 0.f) o[e][i] = __uint_as_float(0x7FC00000u);
          if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  };
  // One piece; lane's tokens are 8 (i / 4) + 4 hh + i % 4.  Only pieces that reach
  // past the tile's first row are masked (those whose NaN values the stash took
  // out): a variant of their own, as selects for all cost a fifth of a step.
  auto block = [&](auto masked_, int buf, int t0) {
    constexpr bool masked = decltype(masked_)::value;
    f32x16_t st;
#pragma unroll
    for (int i = 0; i < 16; ++i) st[i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, sK[buf][2 * kk + hh][c32]);
#pragma unroll
      for (int n = 0; n < QP; ++n) st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[kk][n], st, 0, 0, 0);
    }
    if constexpr (masked) {
      const int left = limit - t0 - 4 * hh;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (8 * (i / 4) + i % 4 >= left) st[i] = -INFINITY;
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // all compares at once spill scalar registers
      }
    }
    float mx = st[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, st[i]);
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
#pragma unroll
    for (int a = 0; a < 2; ++a) {   // 16 tokens
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(st[8 * a + e], sc, -ms));
        l += p[e];
      }
      bf16x8_t pf[PP];
      operand8<PP>(p, pf);
#pragma unroll
      for (int e = 0; e < DT; ++e) {
        const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, sV[buf][a][hh][e][c32]);
#pragma unroll
        for (int n = 0; n < PP; ++n) o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[n], o[e], 0, 0, 0);
      }
    }
    if constexpr (masked)
      if (BOTH ? sNan[buf][0] | sNan[buf][1] | sNan[buf][2] | sNan[buf][3] : sNan[buf][2] | sNan[buf][3]) nan_values(t0);
  };

  if (c0 < c1) {
    auto turn = [&](Load& x, int buf, int t0) {
      stash(x, buf, t0);
      __syncthreads();              // the piece is in LDS; the other buffer is free
      if (t0 + 32 * DEPTH < c1) {
        fetch(x);
        list(t0 + 32 * DEPTH + 32);
      }
      if (active && t0 < wmax) {
        if (t0 + 32 <= whole) block(std::false_type{}, buf, t0);
        else block(std::true_type{}, buf, t0);
      }
    };
    list(c0);
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      fetch(ld[i]);
      list(c0 + 32 * i + 32);
    }
    for (int t0 = c0; t0 < c1; t0 += 64) {
      turn(ld[0], 0, t0);
      if (t0 + 32 < c1) turn(ld[DEPTH - 1], 1, t0 + 32);
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
// One workgroup per (row, head).  The chunks' weights exp2(m_c - M) go to LDS
// first, so that the outputs' loads do not wait for one another; a thread sums 4
// dims over every (1024 / HD)-th chunk, and the threads of a dim join in order.
constexpr int KV8_MAX_SPLIT = 1024;

template <int HD, int OUT>
__global__ __launch_bounds__(256) void k_kv8_merge(Kv8Attn A) {
  constexpr int NT = HD / 4, NG = 256 / NT;   // threads of a chunk's output, chunks side by side
  __shared__ float sw[KV8_MAX_SPLIT], red[16];
  __shared__ __attribute__((aligned(16))) float sO[NG][HD];
  const int r = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  int s, pos;
  if (!kv8_row(A.b, r, s, pos)) return;
  const int ctx = min(pos + 1, kv8_most(A.c, A.b));
  const int n = ctx <= 0 ? 0 : min((ctx - 1) / A.plan.chunk + 1, A.plan.n_split);
  const int64_t slot0 = (int64_t)r * A.plan.n_split;
  float m = -INFINITY;
  for (int c = tid; c < n; c += 256) m = fmaxf(m, part_ml(A, slot0 + c, h)[0]);
  const float M = block_max(m, red);
  float l = 0.f;
  for (int c = tid; c < n; c += 256) {
    const float* ml = part_ml(A, slot0 + c, h);
    const float w = __builtin_amdgcn_exp2f(ml[0] - M);   // all -inf: NaN, as the scores were
    sw[c] = w;
    l += w * ml[1];
  }
  const float L = block_sum(l, red);                       // its barriers order sw too
  const int g = tid / NT, d = tid % NT * 4;
  const float* po = A.part_o + (slot0 * A.n_q + h) * HD + d;
  const int64_t step = (int64_t)A.n_q * HD;
  f32x4_t o = f32x4_t{0.f, 0.f, 0.f, 0.f};
  int c = g;
  for (; c + 7 * NG < n; c += 8 * NG) {
    f32x4_t x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const f32x4_t*>(po + (c + i * NG) * step);
#pragma unroll
    for (int i = 0; i < 8; ++i) o += sw[c + i * NG] * x[i];
  }
  for (; c < n; c += NG) o += sw[c] * *reinterpret_cast<const f32x4_t*>(po + c * step);
  *reinterpret_cast<f32x4_t*>(&sO[g][d]) = o;
  __syncthreads();
  if (tid >= NT) return;
  const float inv = n > 0 ? 1.0f / L : 0.f;
  f32x4_t acc = *reinterpret_cast<const f32x4_t*>(&sO[0][d]);
  for (int i = 1; i < NG; ++i) acc += *reinterpret_cast<const f32x4_t*>(&sO[i][d]);
  const float v[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
  put<OUT>(A, r, h, d, v);
}

template <typename T, int HD, int OUT>
hipError_t run(const Kv8Attn& a, hipStream_t st) {
  const int rep = a.n_q / a.c.n_kv;
  if (a.plan.tiles) {
    const int np = KV8_TILE_Q / rep;
    const int64_t tiles = (int64_t)a.b.rows / np + a.b.n_seqs, grid = tiles * a.c.n_kv * a.plan.n_split;
    if (grid > INT32_MAX) return hipErrorInvalidValue;
    return kv8_launch(k_kv8_tiles<T, HD, OUT>, dim3((unsigned)grid), dim3(64 * KV8_WAVES), st, a);
  }
  const int htiles = (rep + 15) / 16;
  const int64_t items = (int64_t)a.b.rows * a.c.n_kv * htiles * a.plan.n_split;
  const int64_t per = a.plan.deal ? ((int64_t)a.b.rows + 7) / 8 * a.c.n_kv * htiles : (items + 7) / 8;
  if (8 * per > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(8 * per));
  if (a.plan.waves == 8) return kv8_launch(k_kv8_rows<T, HD, OUT, 8>, grid, dim3(512), st, a, htiles, (int)per, (int)items);
  return kv8_launch(k_kv8_rows<T, HD, OUT, 4>, grid, dim3(256), st, a, htiles, (int)per, (int)items);
}

template <int HD, int OUT>
hipError_t merge(const Kv8Attn& a, hipStream_t st) {
  return kv8_launch(k_kv8_merge<HD, OUT>, dim3(a.b.rows, a.n_q), dim3(256), st, a);
}

}  // namespace

// Rows or tiles: a tile's 128 query rows pay from four rows on for each sequence that
// has rows.  Rows pass / tiles of bf16 runs, 2 kv heads of 6 query heads, us: 256
// sequences of 600 tokens with 2, 4 and 8 rows each 22/28, 32/29, 54/32; 64 of 10000
// tokens 71/102, 114/108, 227/118.  Sequences without rows do not count where they are
// known: a recompute of 2048 sequences of 2 to 600 tokens behind 512, 4096 rows a
// launch, takes 141/52 (a bf16 pool's 68).  Batches that leave the chip idle either way
// lose by it: 8 sequences of 600 tokens with 4 to 32 rows each 7/21 to 11/23.
//
// Waves of a rows workgroup: eight where one round of a workgroup a CU holds them
// all (a row's chain of steps is then what the launch waits for: 8 rows of 12 heads
// and 600 tokens 5.5 us, with four waves 6.1), else four (512 rows of 2 kv heads and
// 1556 tokens 55 us; with eight, in two rounds, 63).
//
// Chunks cost their partial outputs and the merge's launch (5 us), so a context is
// cut only as far as one round goes: three rows of 95000 tokens and 4 kv heads take
// 37 + 5 us in 21 chunks (252 workgroups), 48 + 5 in 85.  Rows from 2048 tokens on
// (below, the merge costs what it saves: 600 tokens in two chunks 6.1 + 4.2 us),
// tiles from 1024, which take some 30 us per 1000 tokens; chunks of 512 at least.
Kv8Plan kv8_plan(int rows, int n_seqs, bool has_off, bool tiles, int n_q, int n_kv, int max_len, int max_split) {
  Kv8Plan p{};
  const int rep = n_q / n_kv;
  p.tiles = has_off && tiles && rep <= KV8_TILE_Q && (int64_t)rows >= 4LL * n_seqs;
  const int64_t wgs = p.tiles ? ((int64_t)rows * rep + KV8_TILE_Q - 1) / KV8_TILE_Q * n_kv
                              : (int64_t)rows * n_kv * ((rep + 15) / 16);
  p.waves = wgs <= 256 ? 8 : 4;
  int64_t n = 1;
  if (max_len >= (p.tiles ? 1024 : 2048)) n = std::min<int64_t>((p.tiles ? 512 : 256) / wgs, max_len / 512);
  n = std::max<int64_t>(1, std::min<int64_t>({n, max_split, KV8_MAX_SPLIT}));
  p.chunk = (int)std::min<int64_t>((((int64_t)max_len + n - 1) / n + 63) / 64 * 64, 1 << 30);
  p.n_split = (int)((max_len + (int64_t)p.chunk - 1) / p.chunk);
  if (p.n_split < 1) p.n_split = 1;
  // By length where there is more than one workgroup a CU to even out, and rows
  // enough that an eighth of them is the same for every XCD.
  if (!has_off && p.waves == 4 && p.n_split == 1 && rows >= 64)
    for (int64_t steps = ((int64_t)max_len + 31) >> 5; steps; steps >>= 1) ++p.deal;
  return p;
}

hipError_t launch_kv8_attention(int dtype, bool planes, const Kv8Attn& a, hipStream_t st) {
  if (a.b.rows <= 0 || a.b.n_seqs <= 0) return hipSuccess;
  if ((a.c.hd != 64 && a.c.hd != 128) || a.plan.n_split < 1 || a.plan.n_split > KV8_MAX_SPLIT || a.plan.chunk % 64 ||
      (a.plan.deal && a.b.seq_off) || (a.plan.n_split > 1 && (!a.part_o || !a.part_ml)))
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
