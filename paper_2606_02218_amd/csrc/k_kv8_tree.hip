// Trees of drafted tokens over the 8-bit key/value cache: what each node sees,
// attention of the nodes, and the accepted path's move to its place.
//
// A sequence's last n tokens are its tree's nodes, each behind its parent; node i
// lies in slot context + i of the cache, at position context + depth.  Its mask has
// a bit for itself and every ancestor.
#include <algorithm>
#include <type_traits>

#include "kv8_attn_device.h"

namespace {

// ---------------------------------------------------------------- masks
// A wave a sequence, 64 nodes at a time, a lane each: whoever a node sees of its ancestors it
// passes on, and the reach doubles each time, so six rounds do.  What the 64 see of earlier
// nodes comes from the rows that the wave wrote before.  Latency bound, and by the length alone:
// 8 trees of 130, 500, 2048 nodes take 5, 11, 85 us whatever their shape, 2 of 4096 290.  By walks
// up from each node, n^2 / 128 steps where they are a chain, chains took 58, 424, 6400 us and 25 ms,
// stars 4.5, 8.6, 58 and 176 us.

// Lane `lane`'s node of up to 64, whose parent is lane `up` (-1: none of them): the bits of
// the node and its ancestors among them, and the first of these.  False where it or one of
// them is not `right`.
__device__ __forceinline__ bool tree_bits(int lane, int up, bool right, uint64_t& bits, int& root) {
  int far = right ? up >= 0 ? up : lane : lane | 64;
  bits = 1ull << lane;
#pragma unroll 1
  for (int reach = 1; reach < 64; reach *= 2) {
    const int at = far & 63, next = __shfl(far, at, 64);
    bits |= (uint64_t)__shfl((unsigned long long)bits, at, 64);
    far = next | (far & 64);
  }
  root = far & 63;
  return far < 64;
}

__global__ __launch_bounds__(64) void k_kv8_tree(const int32_t* __restrict__ parent, Kv8Rows b, int words, uint64_t* mask,
                                                 int32_t* pos) {
  const int s = blockIdx.x, lane = threadIdx.x;
  int r0, n;
  kv8_seq_rows(b, s, r0, n);
  if (n <= 0) return;
  const int first = max(n - kv8_len(b, s), 0);          // nodes before it are padding
  const int ctx = max(kv8_len(b, s) - n, 0);
  int next = lane < n ? parent[r0 + lane] : -1;
  if (n <= 64) {
    uint64_t bits;
    int root;
    // no parent: neither the node nor what is behind it counts
    const bool ok = tree_bits(lane, next >= first ? next : -1, next >= -1 && next < lane && lane >= first, bits, root);
    if (lane >= n) return;
    uint64_t* out = mask + (int64_t)(r0 + lane) * words;
    out[0] = ok ? bits : 0;
    for (int w = 1; w < words; ++w) out[w] = 0;
    pos[r0 + lane] = ok ? (int)min((int64_t)ctx + __popcll(bits) - 1, (int64_t)INT32_MAX) : -1;
    return;
  }
  for (int base = 0;; base += 64) {
    const int i = base + lane, up = next, left = n - base;
    if (left > 64) next = lane < left - 64 ? parent[r0 + i + 64] : -1;
    const int out = up >= first && up < base ? up : -1;
    uint64_t bits;
    int root;
    bool ok = tree_bits(lane, up >= max(first, base) ? up - base : -1, lane < left && up >= -1 && up < i && i >= first, bits, root);
    const int back = __shfl(out, root, 64);             // the ancestor before the 64, if there is one
    const int at = ok && back >= 0 ? pos[r0 + back] : ctx - 1;
    ok = ok && (back < 0 || at >= 0);                   // no earlier one of its ancestors was wrong
    if (lane < left) {
      uint64_t* row = mask + (int64_t)(r0 + i) * words;
      const uint64_t* old = mask + (int64_t)(r0 + max(back, 0)) * words;
      const int known = ok && back >= 0 ? min((back >> 6) + 1, words) : 0;
#pragma unroll 1
      for (int w = 0; w < words; w += 8) {              // eight loads on their way together
        uint64_t x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = w + e < known ? old[w + e] : 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (w + e < words) row[w + e] = ok && w + e == base >> 6 ? x[e] | bits : x[e];
      }
      pos[r0 + i] = ok ? (int)min((int64_t)at + __popcll(bits), (int64_t)INT32_MAX) : -1;
    }
    if (left <= 64) return;
    __syncthreads();                                    // these rows can be read
  }
}

// ---------------------------------------------------------------- attention
// The tree's queries of one kv head, nodes x heads, are packed as columns, 16 or 32 of
// them a workgroup.  Its waves take 32-token steps in turn straight from memory, 16 bytes a
// lane, and join in LDS.
// Scores are formed transposed, S^T = K Q^T, so that a lane ends up with the
// probabilities of one column for just those tokens whose V^T operand it loads.
// Every node sees the context: only steps that reach into the tree are masked.
// What bounds the 16: vector issue, and the caches' lines.  A step of 32 tokens x 16 columns
// x 128 dims is 16 MFMAs, 64 conversions of codes and some 60 others, and a wave's start and
// end weigh as much as eight steps.  64 trees of 4 to 63 nodes over 512 to 4500 tokens, 12
// heads, take 83 us, 1400 clocks of a SIMD a step, vector instructions in 55 % of them and
// MFMAs busy in 18 %; by 32 columns 70.  Tried there: four waves of 16 columns, and two or
// four parts of the tokens, over codes that come straight into LDS once 89 and 93 (the
// longest context's chain, and barriers); keys as e4m3 operands beside queries in two e4m3
// pieces 84; every line of a later step touched ahead 108, of a quarter of the steps 86.
constexpr int WIDE_WAVES = 4;
constexpr int tree_pieces(int size) { return size == 2 ? 1 : 3; }   // bf16 pieces of a query and of a probability
constexpr int tree_waves(int size, int hd) { return size == 2 || hd == 64 ? 4 : 3; }   // of a SIMD, by the registers

// 32 bits of a node's mask from bit b on; bits before 0, the context's, are set.
__device__ __forceinline__ uint32_t mask_window(const uint64_t* m, int words, int b) {
  if (b < 0) return b <= -32 ? ~0u : (uint32_t)(m[0] << -b) | ((1u << -b) - 1u);
  const int w = b >> 6, o = b & 63;
  uint64_t x = w < words ? m[w] >> o : 0;
  if (o > 32 && w + 1 < words) x |= m[w + 1] << (64 - o);
  return (uint32_t)x;
}

// Tokens of a sequence that some node of its tree may see: the nodes, n of them, are its
// last ones, those past the mask have no bit, and there is no walk over what the table
// has not.
__device__ __forceinline__ int tree_tokens(const Kv8Pool& c, const Kv8Rows& b, int len, int n, int words) {
  const int64_t ctx0 = (int64_t)len - n, ctx = ctx0 > 0 ? ctx0 : 0, far = ctx0 + 64 * words;
  int64_t t = far > ctx ? far : ctx;
  if (len < t) t = len;
  const int64_t most = (int64_t)kv8_most(c, b) + 64 * words;
  return (int)(t < most ? t : most);
}

// The sequence whose column groups hold number x: sequence s has its groups of
// 2^shift columns at (first row * rep >> shift) + s and on.  64 candidates a step.
__device__ __forceinline__ int find_group(const Kv8Rows& b, int x, int rep, int shift, int& key) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = b.n_seqs, at = 0;
  auto key_of = [&](int s) { return (int)((int64_t)min(max(b.seq_off[s], 0), b.rows) * rep >> shift) + s; };
  do {
    const int step = (hi - lo + 63) >> 6, s = lo + lane * step;
    int k = INT32_MAX;
    if (s < hi) k = key_of(s);
    const uint64_t below = __ballot(s < hi && k <= x) | 1;
    const int top = 63 - __clzll((long long)below);
    at = __builtin_amdgcn_readlane(k, top);
    lo += top * step;
    hi = min(lo + step, hi);
  } while (hi - lo > 1);
  key = at;
  return lo;
}

// The sequence of up to 64 whose column groups hold number x, the longest first: those that
// take longest are not left for the end.  -1: none has it; key: its first group.  A lane a
// sequence, every wave of the workgroup compares with some of them.
template <int W>
__device__ __forceinline__ int find_group_sorted(const Kv8Rows& b, int x, int rep, int shift, int (&sum)[W][64], int& key) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  int r0 = 0, n = 0, len = -1;
  if (lane < b.n_seqs) {
    kv8_seq_rows(b, lane, r0, n);
    len = kv8_len(b, lane);
  }
  const int groups = n > 0 ? (int)(((int64_t)n * rep + (1 << shift) - 1) >> shift) : 0;
  int first = 0;
  for (int t = wave; t < b.n_seqs; t += W) {
    const int l = __builtin_amdgcn_readlane(len, t), g = __builtin_amdgcn_readlane(groups, t);
    first += l > len || (l == len && t < lane) ? g : 0;
  }
  sum[wave][lane] = first;
  __syncthreads();
  first = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) first += sum[w][lane];
  const uint64_t here = __ballot(x >= first && x < first + groups);
  if (!here) return -1;
  const int s = __ffsll((unsigned long long)here) - 1;
  key = __builtin_amdgcn_readlane(first, s);
  return s;
}

// The largest of a lane's scores; NaN where one is: it stays out of the running maximum.
__device__ __forceinline__ float top8(const f32x4_t (&s)[2]) {
  auto most = [](float a, float b) { return __builtin_elementwise_maximum(a, b); };
  return most(most(most(s[0][0], s[0][1]), most(s[0][2], s[0][3])), most(most(s[1][0], s[1][1]), most(s[1][2], s[1][3])));
}

// Eight probabilities as operands, and their sum: of bf16 ones as they enter the product
// (2 of 64 nodes over 60 to 131 thousand tokens 200 us, by additions beforehand 214).
template <int N>
__device__ __forceinline__ void weigh8(const float (&p)[8], bf16x8_t (&out)[N], float& l) {
  operand8<N>(p, out);
  if constexpr (N == 1) {
    typedef __bf16 pair_t __attribute__((ext_vector_type(2)));
    const u32x4_t w = __builtin_bit_cast(u32x4_t, out[0]);
    const pair_t ones = __builtin_bit_cast(pair_t, 0x3F803F80u);
#pragma unroll
    for (int e = 0; e < 4; ++e) l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair_t, (uint32_t)w[e]), ones, l, false);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) l += p[e];
  }
}

// Whether a row, node of its sequence, sees any of the tokens c0 .. c1 - 1.
__device__ __forceinline__ bool sees_any(const Kv8Attn& A, int row, int node, int ctx0, int c0, int c1) {
  if (ctx0 + node < 0) return false;
  if (c0 < min(ctx0, c1)) return true;
  for (int t = max(c0, max(ctx0, 0)); t < c1; t += 32) {
    const uint32_t bits = mask_window(A.mask + (int64_t)row * A.words, A.words, t - ctx0);
    if (c1 - t < 32 ? bits & ((1u << (c1 - t)) - 1u) : bits) return true;
  }
  return false;
}
// A sum of weights that is -0 is that of no tokens: what sees some, all with a score of -inf,
// has +0 and its output is 0 / 0.
__device__ __forceinline__ bool is_none(float sum) { return __float_as_uint(sum) == 0x80000000u; }

// N dims of column c from d on: the waves' results joined, NaN values of the tokens that its
// node does see put back, and stored, or kept for the join of the chunks.  Steps that reach
// into the tree cleared them, so the first token to look at is that of the step with the
// first node, which may hold up to 31 of the context's (chunks begin at whole steps).
template <typename T, int HD, int W, int N>
__device__ __forceinline__ void tree_store(const Kv8Attn& A, const float (&ml)[W], const float (&sum)[W],
                                           const float* (&acc)[W], uint32_t c, int d, int rep, int kvh, int r0, int ctx0, int split,
                                           int c0, int c1, bool fix, const int32_t* tab) {
  const int node = (int)(c / (uint32_t)rep), head = kvh * rep + (int)(c - (uint32_t)node * rep);
  float M = ml[0];
#pragma unroll
  for (int w = 1; w < W; ++w) M = fmaxf(M, ml[w]);
  float L = 0.f, o[N];
#pragma unroll
  for (int e = 0; e < N; ++e) o[e] = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) {                         // a wave without steps has weight 0
    const float f = ml[w] == M ? 1.f : __builtin_amdgcn_exp2f(ml[w] - M);
    L += f * sum[w];
    float x[N];
    ld_elems<N, true>(acc[w] + d, x);
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] += f * x[e];
  }
  if (fix && ctx0 + node >= 0) {
    const uint64_t* mask = A.mask + (int64_t)(r0 + node) * A.words;
    for (int t = max(max(ctx0, 0) & ~31, c0); t < c1; ++t) {
      if (!(mask_window(mask, A.words, t - ctx0) & 1)) continue;
      const int b = kv8_block(A.c, tab, A.b.tab_stride, t >> 4, kvh);
      if (b < 0) continue;                              // its scores are NaN
      const uint8_t* v = A.c.v + (int64_t)b * (16 * HD) + (t >> 2 & 3) * (4 * HD) + d * 4 + (t & 3);
#pragma unroll
      for (int e = 0; e < N; ++e)
        if ((v[4 * e] & 0x7F) == 0x7F) o[e] = __uint_as_float(0x7FC00000u);
    }
  }
  if (L == 0.f && !sees_any(A, r0 + node, node, ctx0, c0, c1)) L = -0.f;
  if (A.plan.n_split == 1) {
    const float inv = is_none(L) ? 0.f : 1.0f / L;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] *= inv;
    st_elems<N, true>((T*)A.out + ((int64_t)(r0 + node) * A.n_q + head) * HD + d, o);
  } else {
    const int64_t slot = ((int64_t)(r0 + node) * A.plan.n_split + split) * A.n_q + head;
    if (c0 < c1) st_elems<N, true>(A.part_o + slot * HD + d, o);
    if (d == 0) {
      A.part_ml[2 * slot] = M;
      A.part_ml[2 * slot + 1] = L;
    }
  }
}

template <typename T, int HD, int W>
__global__ __launch_bounds__(64 * W, tree_waves(sizeof(T), HD)) void k_kv8_tree_attn(Kv8Attn A, unsigned eights,
                                                                                      unsigned items) {
  constexpr int QP = tree_pieces(sizeof(T)), PP = QP;
  constexpr int NJ = HD / 64;       // 16-byte loads of a block per lane
  constexpr int LDO = HD + 4;
  __shared__ __attribute__((aligned(16))) float sO[W][16][LDO];
  __shared__ float sM[W][16], sL[W][16];
  __shared__ int sNan[W], sFind[W][64];

  // Blocks are dealt to the 8 XCDs in turn; runs of eight items, column groups that
  // read the same tokens, stay on one.
  unsigned item = (blockIdx.x >> 6) * 64 + (blockIdx.x & 7) * 8 + (blockIdx.x >> 3 & 7);
  if (item >= items) return;
  // eight groups, then those of the other kv heads, then the next eight; chunk after chunk
  unsigned run = item >> 3;
  const int kvh = (int)(run % (unsigned)A.c.n_kv);
  run /= (unsigned)A.c.n_kv;
  const int split = (int)(run / eights), x = (int)(run - (unsigned)split * eights) * 8 + (int)(item & 7);
  const int rep = A.n_q / A.c.n_kv;
  int key = 0, r0, n;
  // where one round of workgroups does not hold them all the order counts
  const int s = A.b.n_seqs <= 64 && gridDim.x > 256 ? find_group_sorted(A.b, x, rep, 4, sFind, key) : find_group(A.b, x, rep, 4, key);
  if (s < 0) return;
  kv8_seq_rows(A.b, s, r0, n);
  const uint32_t cols = (uint32_t)n * rep, col0 = (uint32_t)(x - key) * 16;   // each an output row's head: below 2^32
  if (x < key || col0 >= cols) return;
  const int len = kv8_len(A.b, s), ctx0 = len - n;      // node i is token ctx0 + i
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cl = lane & 15, grp = lane >> 4;
  const int total = tree_tokens(A.c, A.b, len, n, A.words);   // those that some node may see
  const int64_t c0l = (int64_t)split * A.plan.chunk;
  const int c0 = (int)std::min<int64_t>(c0l, total);
  const int c1 = split == A.plan.n_split - 1 ? total : (int)std::min<int64_t>(total, c0l + A.plan.chunk);
  const int steps = (c1 - c0 + 31) / 32, last_blk = (max(c1, 1) - 1) >> 4;
  const int mine = (steps - wave + W - 1) / W;          // steps wave, wave + W, ...
  const int whole = min(max(ctx0, 0), c1);              // tokens that every node sees
  const int32_t* tab = kv8_table(A.b, s);

  const uint8_t* kl = A.c.k + lane * 16;
  const uint8_t* vl = A.c.v + grp * (4 * HD) + cl * 16;
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
      for (int j = 0; j < NJ; ++j) kr[h][j] = *reinterpret_cast<const u32x4_t*>(p + j * 1024);
    }
  };
  auto fetch_v = [&](int i) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* p = vl + (int64_t)max(__builtin_amdgcn_readlane(ids, 2 * (i & 31) + h), 0) * (16 * HD);
#pragma unroll
      for (int j = 0; j < NJ; ++j) vr[h][j] = *reinterpret_cast<const u32x4_t*>(p + j * 256);
    }
  };
  if (mine > 0) {                   // on their way beside the queries
    lists(0);
    fetch_k(0);
    fetch_v(0);
  }

  const float sc = A.scale * KV8_LOG2E;
  float m = -INFINITY, l = 0.f;
  f32x4_t o[NJ][4];
  bf16x8_t qf[2 * NJ][QP];
  const bool vec = (((uintptr_t)A.q.p | (A.q.row * sizeof(T)) | (A.q.head * sizeof(T))) & 15) == 0;
  const uint32_t c = col0 + cl;
  const bool valid = c < cols;
  const int node = valid ? (int)(c / (uint32_t)rep) : 0, head = kvh * rep + (valid ? (int)(c - (uint32_t)node * rep) : 0);
  const int row = valid && ctx0 + node >= 0 ? r0 + node : -1;   // -1: the column sees nothing, as padding, or is none
  const T* qp = (const T*)A.q.p + max(row, 0) * A.q.row + head * A.q.head;
#pragma unroll
  for (int kk = 0; kk < 2 * NJ; ++kk) query8<T, QP>(qp + 64 * (kk >> 1) + 16 * grp + 8 * (kk & 1), row >= 0, vec, qf[kk]);
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[j][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  bool nan = false;                 // values of the tree's tokens that are NaN

  for (int i = 0; i < mine; ++i) {
    const int t0 = c0 + 32 * (wave + W * i);
    float vs[2];
    int id[2];
    f32x4_t st[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      id[h] = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + h);
      const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(kss), 2 * (i & 31) + h));
      vs[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vss), 2 * (i & 31) + h));
      // a lost page's tokens: NaN scores (the codes in the registers are another page's)
      const float none = id[h] < 0 ? __uint_as_float(0x7FC00000u) : 0.f;
      st[h] = f32x4_t{none, none, none, none};
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bf16x8_t kf = kv8_bf16x8(kr[h][j][2 * e], kr[h][j][2 * e + 1], ks, ks);
#pragma unroll
          for (int n_ = 0; n_ < QP; ++n_)
            st[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[2 * j + e][n_], st[h], 0, 0, 0);
        }
    }
    // the next step's keys into the registers just read: they arrive under the softmax
    // and the values' products, and other waves' work
    if (i + 1 < mine) {
      if (((i + 1) & 31) == 0) lists(i + 1);
      fetch_k(i + 1);
    }
    // lane's tokens: 16 h + 4 grp + e of the step
    if (t0 + 32 > whole) {
      const uint32_t there = c1 - t0 < 32 ? (1u << (c1 - t0)) - 1u : ~0u;
      uint32_t seen = 0;
      if (row >= 0) seen = mask_window(A.mask + (int64_t)row * A.words, A.words, t0 - ctx0) & there;
      seen >>= 4 * grp;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!(seen >> (16 * h + e) & 1)) st[h][e] = -INFINITY;
      // 0 * NaN is NaN: what some column does not see must hold none.  Stale slots and lost
      // pages are cleared, and NaN codes, which the end looks after.
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int left = id[h] < 0 ? 0 : min(max(c1 - t0 - 16 * h - 4 * grp, 0), 4);
        const uint32_t keep = left == 4 ? ~0u : (1u << (8 * left)) - 1u;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t w = vr[h][j][e] & keep;
            nan |= has_nan_code(w);
            vr[h][j][e] = clear_nan(w);
          }
      }
    }
    bf16x8_t pf[PP];
    float mx = top8(st) * sc;
    if (__any(mx > m + KV8_SLACK)) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = fmaxf(m, mx);
      const float alpha = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);   // -inf: nothing seen yet
      l *= alpha;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] *= alpha;
      m = mn;
    }
    const float ms = m == -INFINITY ? 0.f : m;   // nothing seen: every probability is exp2(-inf) = 0
    float p[8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) p[4 * h + e] = __builtin_amdgcn_exp2f(fmaf(st[h][e], sc, -ms));
    weigh8<PP>(p, pf, l);
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bf16x8_t vf = kv8_bf16x8(vr[0][j][e], vr[1][j][e], vs[0], vs[1]);
#pragma unroll
        for (int n_ = 0; n_ < PP; ++n_)
          o[j][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n_], o[j][e], 0, 0, 0);
      }
    if (i + 1 < mine) fetch_v(i + 1);
  }

  // Join the waves: column cl, dims 64 j + 16 grp + 4 i + e of
  // the lane.  A wave without steps has weight 0.
  const bool any_nan = __any(nan);
  if (lane == 0) sNan[wave] = any_nan;
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (grp == 0) {
    sM[wave][cl] = m;
    sL[wave][cl] = l;
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4_t*>(&sO[wave][cl][64 * j + 16 * grp + 4 * i]) =
          f32x4_t{o[j][0][i], o[j][1][i], o[j][2][i], o[j][3][i]};
  __syncthreads();
  bool fix = false;
#pragma unroll
  for (int w = 0; w < W; ++w) fix |= sNan[w] != 0;
  constexpr int N = 16 * HD / (64 * W);
  const int h = tid / (HD / N), d = tid % (HD / N) * N;
  if (col0 + h >= cols) return;
  float ml[W], sum[W];
  const float* acc[W];
#pragma unroll
  for (int w = 0; w < W; ++w) {
    ml[w] = sM[w][h];
    sum[w] = sL[w][h];
    acc[w] = sO[w][h];
  }
  tree_store<T, HD, W, N>(A, ml, sum, acc, col0 + h, d, rep, kvh, r0, ctx0, split, c0, c1, fix, tab);
}

// The same for 32 columns a workgroup: a step's codes pass the caches and are converted
// once for twice as many.  The queries' operands come through LDS, where the waves share
// them.
// What bounds it: matrix and vector issue.  A step of 32 tokens and 128 dims is 16 products of
// 32 x 32 x 16, which hold the vector unit for half of their 32 clocks each, and 64
// conversions, 16 exponentials and some 80 others.  64 trees of 64 nodes, 12 heads, at 4000
// tokens 154 us, 0.66 PFLOP/s; 2 of 64, 28 heads, at 60 to 131 thousand 200 (0.67), vector
// instructions in 52 % of the cycles, MFMAs busy in 31 %.
template <typename T, int HD>
__global__ __launch_bounds__(64 * WIDE_WAVES, sizeof(T) == 2 ? 3 : 2) void k_kv8_tree_wide(Kv8Attn A, unsigned eights,
                                                                                            unsigned items) {
  constexpr int QP = tree_pieces(sizeof(T)), PP = QP, W = WIDE_WAVES;
  constexpr int NK = HD / 16;       // products over the head's dims
  constexpr int NL = HD / 32;       // 16-byte loads of a step's keys per lane
  constexpr int DT = HD / 32;       // 32-dim tiles of the output: tile e holds dims DT * row + e
  constexpr int LDO = HD + 4;
  union Memory {
    u32x4_t q[NK][QP][2][32];       // [product][piece][half][column]
    float o[W][16][LDO];
  };
  __shared__ Memory mem;
  __shared__ float sM[W][32], sL[W][32];
  __shared__ int sNan[W], sFind[W][64];

  unsigned item = (blockIdx.x >> 6) * 64 + (blockIdx.x & 7) * 8 + (blockIdx.x >> 3 & 7);
  if (item >= items) return;
  unsigned run = item >> 3;
  const int kvh = (int)(run % (unsigned)A.c.n_kv);
  run /= (unsigned)A.c.n_kv;
  const int split = (int)(run / eights), x = (int)(run - (unsigned)split * eights) * 8 + (int)(item & 7);
  const int rep = A.n_q / A.c.n_kv;
  int key = 0, r0, n;
  const int s =
      A.b.n_seqs <= 64 && gridDim.x > 256 ? find_group_sorted(A.b, x, rep, 5, sFind, key) : find_group(A.b, x, rep, 5, key);
  if (s < 0) return;
  kv8_seq_rows(A.b, s, r0, n);
  const uint32_t cols = (uint32_t)n * rep, col0 = (uint32_t)(x - key) * 32;
  if (x < key || col0 >= cols) return;
  const int len = kv8_len(A.b, s), ctx0 = len - n;      // node i is token ctx0 + i
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c32 = lane & 31, hh = lane >> 5;
  const int total = tree_tokens(A.c, A.b, len, n, A.words);
  const int64_t c0l = (int64_t)split * A.plan.chunk;
  const int c0 = (int)std::min<int64_t>(c0l, total);
  const int c1 = split == A.plan.n_split - 1 ? total : (int)std::min<int64_t>(total, c0l + A.plan.chunk);
  const int steps = (c1 - c0 + 31) / 32, last_blk = (max(c1, 1) - 1) >> 4;
  const int mine = (steps - wave + W - 1) / W;
  const int whole = min(max(ctx0, 0), c1);
  const int32_t* tab = kv8_table(A.b, s);

  // Keys: lane c32 a token, 16 dims of every other 32; values: dims DT c32 .. of the
  // token quads hh and 2 + hh of both blocks.
  const uint8_t* kl = A.c.k + hh * 256 + (c32 & 15) * 16;
  const uint8_t* vl = A.c.v + hh * (4 * HD) + c32 * (4 * DT);
  typedef uint32_t vals_t __attribute__((ext_vector_type(DT)));
  u32x4_t kr[NL];
  vals_t vr[2][2];
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
    const int i0 = __builtin_amdgcn_readlane(ids, 2 * (i & 31)), i1 = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + 1);
    const uint8_t* p = kl + (int64_t)max(c32 < 16 ? i0 : i1, 0) * (16 * HD);
#pragma unroll
    for (int j = 0; j < NL; ++j) kr[j] = *reinterpret_cast<const u32x4_t*>(p + j * 512);
  };
  auto fetch_v = [&](int i) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* p = vl + (int64_t)max(__builtin_amdgcn_readlane(ids, 2 * (i & 31) + h), 0) * (16 * HD);
#pragma unroll
      for (int g = 0; g < 2; ++g) vr[h][g] = *reinterpret_cast<const vals_t*>(p + g * (8 * HD));
    }
  };
  if (mine > 0) {
    lists(0);
    fetch_k(0);
    fetch_v(0);
  }
  const bool vec = (((uintptr_t)A.q.p | (A.q.row * sizeof(T)) | (A.q.head * sizeof(T))) & 15) == 0;
  for (int i = tid; i < NK * 64; i += 64 * W) {         // the columns' queries
    const int kk = i >> 6, half = i >> 5 & 1, cc = i & 31;
    const uint32_t c = col0 + cc;
    const int node = (int)(c / (uint32_t)rep), head = kvh * rep + (int)(c - (uint32_t)node * rep);
    const bool ok = c < cols && ctx0 + node >= 0;
    bf16x8_t f[QP];
    const T* at = (const T*)A.q.p + (r0 + (ok ? node : 0)) * A.q.row + head * A.q.head;
    query8<T, QP>(at + 16 * ((kk & ~1) + half) + 8 * (kk & 1), ok, vec, f);
#pragma unroll
    for (int p = 0; p < QP; ++p) mem.q[kk][p][half][cc] = __builtin_bit_cast(u32x4_t, f[p]);
  }
  const uint32_t c = col0 + c32;
  const int node_ = (int)(c / (uint32_t)rep);
  const int row = c < cols && ctx0 + node_ >= 0 ? r0 + node_ : -1;   // -1: the column sees nothing
  const float sc = A.scale * KV8_LOG2E;
  float m = -INFINITY, l = 0.f;
  f32x16_t o[DT];
#pragma unroll
  for (int e = 0; e < DT; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[e][i] = 0.f;
  bool nan = false;
  __syncthreads();

  for (int i = 0; i < mine; ++i) {
    const int t0 = c0 + 32 * (wave + W * i);
    int id[2];
    float ks[2], vs[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      id[h] = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + h);
      ks[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(kss), 2 * (i & 31) + h));
      vs[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vss), 2 * (i & 31) + h));
    }
    const float kscale = c32 < 16 ? ks[0] : ks[1];
    f32x16_t st;                    // lane's tokens: 8 (i / 4) + 4 hh + i % 4 of the step
#pragma unroll
    for (int e = 0; e < 16; ++e) st[e] = id[e >> 3] < 0 ? __uint_as_float(0x7FC00000u) : 0.f;   // a lost page's: NaN
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      const bf16x8_t kf = kv8_bf16x8(kr[kk >> 1][2 * (kk & 1)], kr[kk >> 1][2 * (kk & 1) + 1], kscale, kscale);
#pragma unroll
      for (int p = 0; p < QP; ++p)
        st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, __builtin_bit_cast(bf16x8_t, mem.q[kk][p][hh][c32]), st, 0, 0, 0);
    }
    if (i + 1 < mine) {
      if (((i + 1) & 31) == 0) lists(i + 1);
      fetch_k(i + 1);
    }
    if (t0 + 32 > whole) {
      const uint32_t there = c1 - t0 < 32 ? (1u << (c1 - t0)) - 1u : ~0u;
      uint32_t seen = 0;
      if (row >= 0) seen = mask_window(A.mask + (int64_t)row * A.words, A.words, t0 - ctx0) & there;
      seen >>= 4 * hh;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!(seen >> (8 * (e / 4) + e % 4) & 1)) st[e] = -INFINITY;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const int left = id[h] < 0 ? 0 : min(max(c1 - t0 - 16 * h - 8 * g - 4 * hh, 0), 4);
          const uint32_t keep = left == 4 ? ~0u : (1u << (8 * left)) - 1u;
#pragma unroll
          for (int e = 0; e < DT; ++e) {
            const uint32_t w = vr[h][g][e] & keep;
            nan |= has_nan_code(w);
            vr[h][g][e] = clear_nan(w);
          }
        }
    }
    float mx = st[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = __builtin_elementwise_maximum(mx, st[e]);
    mx *= sc;
    if (__any(mx > m + KV8_SLACK)) {
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = fmaxf(m, mx);
      const float alpha = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      l *= alpha;
#pragma unroll
      for (int e = 0; e < DT; ++e) o[e] *= alpha;
      m = mn;
    }
    const float ms = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int h = 0; h < 2; ++h) {   // 16 tokens
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(st[8 * h + e], sc, -ms));
      bf16x8_t pf[PP];
      weigh8<PP>(p, pf, l);
#pragma unroll
      for (int e = 0; e < DT; ++e) {
        const bf16x8_t vf = kv8_bf16x8(vr[h][0][e], vr[h][1][e], vs[h], vs[h]);
#pragma unroll
        for (int q = 0; q < PP; ++q) o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[q], o[e], 0, 0, 0);
      }
    }
    if (i + 1 < mine) fetch_v(i + 1);
  }

  const bool any_nan = __any(nan);
  if (lane == 0) sNan[wave] = any_nan;
  l += __shfl_xor(l, 32, 64);
  if (hh == 0) {
    sM[wave][c32] = m;
    sL[wave][c32] = l;
  }
  bool fix = false;
  for (int half = 0; half < 2; ++half) {                // 16 columns at a time: dims DT * (8 (i / 4) + 4 hh + i % 4) + e
    __syncthreads();                                    // the queries, or the other half, have been read
    if (c32 >> 4 == half) {
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < DT; ++e) mem.o[wave][c32 & 15][DT * (8 * g + 4 * hh + i) + e] = o[e][4 * g + i];
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) fix |= sNan[w] != 0;
    constexpr int N = 16 * HD / (64 * W);
    const int h = 16 * half + tid / (HD / N), d = tid % (HD / N) * N;
    if (col0 + h < cols) {
      float ml[W], sum[W];
      const float* acc[W];
#pragma unroll
      for (int w = 0; w < W; ++w) {
        ml[w] = sM[w][h];
        sum[w] = sL[w][h];
        acc[w] = mem.o[w][h & 15];
      }
      tree_store<T, HD, W, N>(A, ml, sum, acc, col0 + h, d, rep, kvh, r0, ctx0, split, c0, c1, fix, tab);
    }
  }
}

// A wave per row and head joins the chunks' partial results in order; a chunk that
// the row sees nothing of has sum 0 and its outputs are not looked at.
constexpr int TREE_MAX_SPLIT = 64;

template <typename T, int HD>
__global__ __launch_bounds__(256) void k_kv8_tree_merge(Kv8Attn A) {
  constexpr int ND = HD / 64;
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int64_t r = at / A.n_q;
  const int head = (int)(at - r * A.n_q);
  if (r >= A.b.rows || r < A.b.seq_off[0] || r >= A.b.seq_off[A.b.n_seqs]) return;
  const int64_t slot0 = r * A.plan.n_split * A.n_q + head;
  float m = -INFINITY, l = -0.f;
  if (lane < A.plan.n_split) {
    const float* ml = A.part_ml + 2 * (slot0 + (int64_t)lane * A.n_q);
    m = ml[0];
    l = ml[1];
  }
  const float M = wave_max(m);
  const float w = l == 0.f ? 0.f : m == M ? 1.f : __builtin_amdgcn_exp2f(m - M);
  const float L = wave_sum(w * l), inv = __all(is_none(l)) ? 0.f : 1.0f / L;
  float acc[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) acc[i] = 0.f;
  for (uint64_t some = __ballot(l != 0.f); some; some &= some - 1) {   // NaN sums too
    const int c = __ffsll((unsigned long long)some) - 1;
    const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), c));
    const float* o = A.part_o + (slot0 + (int64_t)c * A.n_q) * HD + lane * ND;
#pragma unroll
    for (int i = 0; i < ND; ++i) acc[i] += f * o[i];
  }
#pragma unroll
  for (int i = 0; i < ND; ++i) acc[i] *= inv;
  T* out = (T*)A.out + at * HD + lane * ND;
  if constexpr (ND == 2 && sizeof(T) == 2) *reinterpret_cast<uint32_t*>(out) = pack_bf16x2(acc[0], acc[1]);
  else st_elems<ND, false>(out, acc);
}

// ---------------------------------------------------------------- accepted paths
// The j-th kept node moves to slot ctx + j, which no later kept node comes from: a
// destination block reads its own slots or ones behind them.  A workgroup per
// sequence, kv head and keys or values: each wave gathers one block, all of them
// wait, then store, so that no store passes a load of a round, and later rounds read
// behind what earlier ones wrote.  A block's scale is the largest of the tokens that
// end up in it, a power of two, so that a moved code keeps its bits unless it lands
// among the subnormals.
constexpr int ACCEPT_WAVES = 4;

struct AcceptArgs {
  Kv8Pool c;
  Kv8Rows b;
  const uint64_t* mask;
  int words;
  const int32_t* last;
  int32_t* new_len;
};

// Word w of the kept nodes: those that are in the cache and among the n.
__device__ __forceinline__ uint64_t kept_word(const uint64_t* m, int w, int first, int n) {
  uint64_t x = m[w];
  const int lo = first - 64 * w, hi = n - 64 * w;
  if (lo > 0) x = lo >= 64 ? 0 : x & ~0ull << lo;
  if (hi < 64) x = hi <= 0 ? 0 : x & ~0ull >> (64 - hi);
  return x;
}

// Index of the k-th set bit of x (one that has more than k).
__device__ __forceinline__ int nth_bit(uint64_t x, int k) {
  int at = 0;
#pragma unroll
  for (int half = 32; half > 0; half >>= 1) {
    const int c = __popcll(x & ((1ull << half) - 1));
    if (k >= c) { k -= c; x >>= half; at += half; }
  }
  return at;
}

template <int HD>
__global__ __launch_bounds__(64 * ACCEPT_WAVES) void k_kv8_accept(AcceptArgs A) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  unsigned item = blockIdx.x;
  const bool values = item & 1;
  item >>= 1;
  const int s = (int)(item / (unsigned)A.c.n_kv), kvh = (int)(item - (unsigned)s * A.c.n_kv);
  int r0, n;
  kv8_seq_rows(A.b, s, r0, n);
  const int len = kv8_len(A.b, s), ctx0 = len - n, ctx = max(ctx0, 0), first = max(-ctx0, 0);
  const int last = n > 0 ? A.last[s] : -1;
  const bool some = last >= 0 && last < n;
  const uint64_t* mask = A.mask + (int64_t)(some ? r0 + last : 0) * A.words;
  int kept = 0, stay = 0;                                // kept nodes; those before the first gap
  if (some) {
    bool gap = false;
    for (int w = 0; w < A.words; ++w) {
      const uint64_t x = kept_word(mask, w, first, n);
      kept += __popcll(x);
      if (!gap) {
        const uint64_t y = w == first >> 6 ? x >> (first & 63) : w < first >> 6 ? ~0ull : x;
        const int run = w < first >> 6 ? 0 : ~y ? __ffsll((unsigned long long)~y) - 1 : 64;
        stay += run;
        gap = w >= first >> 6 && run < 64 - (w == first >> 6 ? first & 63 : 0);
      }
    }
  }
  const int end = ctx + kept;
  if (kvh == 0 && !values && threadIdx.x == 0) A.new_len[s] = end;
  if (stay == kept) return;                              // nothing moves
  const int32_t* tab = kv8_table(A.b, s);
  uint8_t* codes = values ? A.c.v : A.c.k;
  float* scales = values ? A.c.v_scale : A.c.k_scale;
  const int b0 = (ctx + stay) >> 4, b1 = (end - 1) >> 4;
  for (int base = b0; base <= b1; base += ACCEPT_WAVES) {
    const int blk = base + wave;
    const bool on = blk <= b1;
    // token t of the block: where it is now
    const int t = lane & 15, p = 16 * blk + t;
    int src = p;
    const bool there = on && p < end;
    if (there && p >= ctx + stay) {
      int j = p - ctx;
      for (int w = 0; w < A.words; ++w) {
        const uint64_t x = kept_word(mask, w, first, n);
        const int c = __popcll(x);
        if (j < c) { src = ctx0 + 64 * w + nth_bit(x, j); break; }
        j -= c;
      }
    }
    int from = -1;
    float scale = 0.f;
    if (there) {
      from = kv8_block(A.c, tab, A.b.tab_stride, src >> 4, kvh);
      if (from >= 0) scale = scales[from];
    }
    const int to = on ? kv8_block(A.c, tab, A.b.tab_stride, blk, kvh) : -1;
    float top = scale;
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    if (!(top > 0.f)) top = 1.f;                         // pages that are not there: the codes become NaN
    const float ratio = from < 0 ? __uint_as_float(0x7FC00000u) : scale / top;
    // what the tokens that end up here hold, as they are
    u32x4_t kd[HD / 64];
    uint32_t vd[4][HD / 16];
    const int kt = lane >> 2, kc = lane & 3;             // keys: four lanes a token
    const int vq = lane >> 4, vd0 = (lane & 15) * (HD / 16);   // values: four tokens of some dims
    if (!values) {
      const int f = max(__shfl(from, kt, 64), 0), ts = __shfl(src, kt, 64) & 15;
#pragma unroll
      for (int g = 0; g < HD / 64; ++g)
        kd[g] = *reinterpret_cast<const u32x4_t*>(codes + (int64_t)f * (16 * HD) + (kc + 4 * g) * 256 + ts * 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int f = max(__shfl(from, 4 * vq + i, 64), 0), ts = __shfl(src, 4 * vq + i, 64) & 15;
        const uint32_t* w = reinterpret_cast<const uint32_t*>(codes + (int64_t)f * (16 * HD) + (ts >> 2) * (4 * HD)) + vd0;
#pragma unroll
        for (int d = 0; d < HD / 16; d += 4) {
          const u32x4_t z = *reinterpret_cast<const u32x4_t*>(w + d);
#pragma unroll
          for (int e = 0; e < 4; ++e) vd[i][d + e] = z[e] >> (8 * (ts & 3)) & 0xFFu;
        }
      }
    }
    __syncthreads();                                     // every load of the round is in registers
    if (to >= 0) {
      uint8_t* out = codes + (int64_t)to * (16 * HD);
      if (!values) {
        const float f = __shfl(ratio, kt, 64);
        if (__shfl((int)there, kt, 64)) {
#pragma unroll
          for (int g = 0; g < HD / 64; ++g) {
            u32x4_t z;
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = kv8_requant4(kd[g][e], f);
            *reinterpret_cast<u32x4_t*>(out + (kc + 4 * g) * 256 + kt * 16) = z;
          }
        }
      } else {
        float f[4];
        uint32_t fresh = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[i] = __shfl(ratio, 4 * vq + i, 64);
          if (__shfl((int)there, 4 * vq + i, 64)) fresh |= 0xFFu << (8 * i);
        }
        if (fresh) {
          uint32_t* w = reinterpret_cast<uint32_t*>(out + vq * (4 * HD)) + vd0;
#pragma unroll
          for (int d = 0; d < HD / 16; d += 4) {
            u32x4_t z = u32x4_t{0, 0, 0, 0};
            if (fresh != ~0u) z = *reinterpret_cast<const u32x4_t*>(w + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float y[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_cvt_f32_fp8((int)vd[i][d + e], 0) * f[i];
              z[e] = (kv8_codes4(y[0], y[1], y[2], y[3]) & fresh) | (z[e] & ~fresh);
            }
            *reinterpret_cast<u32x4_t*>(w + d) = z;
          }
        }
      }
      if (lane == 0) scales[to] = top;
    }
    __syncthreads();                                     // the next round's loads see none of these slots, but the same scales
  }
}

template <typename T, int HD>
hipError_t run(const Kv8TreeAttn& t, hipStream_t st) {
  const Kv8Attn& a = t.a;
  const int rep = a.n_q / a.c.n_kv;
  const int64_t eights = ((int64_t)a.b.rows * rep / (t.wide ? 32 : 16) + a.b.n_seqs + 7) / 8;
  const int64_t items = eights * 8 * a.c.n_kv * a.plan.n_split;
  if (items > INT32_MAX - 64) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((items + 63) / 64 * 64));
  const unsigned e = (unsigned)eights, n = (unsigned)items;
  if (t.wide) return kv8_launch(k_kv8_tree_wide<T, HD>, grid, dim3(64 * WIDE_WAVES), st, a, e, n);
  if (a.plan.waves == 8) return kv8_launch(k_kv8_tree_attn<T, HD, 8>, grid, dim3(512), st, a, e, n);
  return kv8_launch(k_kv8_tree_attn<T, HD, 4>, grid, dim3(256), st, a, e, n);
}

template <typename T, int HD>
hipError_t merge(const Kv8Attn& a, hipStream_t st) {
  const int64_t n = ((int64_t)a.b.rows * a.n_q + 3) / 4;
  if (n > INT32_MAX) return hipErrorInvalidValue;
  return kv8_launch(k_kv8_tree_merge<T, HD>, dim3((unsigned)n), dim3(256), st, a);
}

}  // namespace

// 32 columns a workgroup where sequences have 64 and more on average and there are, with
// their contexts cut into chunks of 640 tokens and more, workgroups enough: as many as three a
// compute unit (fp32 two), 384 of them at least.  64 trees of 64 nodes, 12 heads, at 4000 tokens
// 154 us, by 16 columns 199; 3 of 40 to 60, 28 heads, at 20 to 25 thousand 101 and 171; but 8
// of 20 to 30, 12 heads, at 1000 to 1500 17 and 12, 48 of 5 to 10 21 and 19.  Else 16
// columns, whose contexts are cut only where that fills the chip, since the chunks' partial
// results and the join's launch cost more than they even out (64 trees of 4 to 63 nodes at
// 512 to 4500 tokens 83 us in one piece, 92 in two), and 8 waves share a workgroup's tokens
// where one round holds them.
Kv8TreePlan kv8_tree_plan(int dtype, int rows, int n_seqs, int n_q, int n_kv, int max_len) {
  Kv8TreePlan p{};
  max_len = std::min(max_len, 1 << 30);                 // a table's most: one chunk, where nothing else asks for more
  const int64_t rep = n_q / n_kv, cols = (int64_t)rows * rep / n_seqs, most = max_len / 640;
  const auto groups = [&](int of) { return ((int64_t)rows * rep / of + n_seqs / 2 + 1) * n_kv; };
  const int64_t wide = groups(32), full = dtype == 1 ? 768 : 512;
  const int64_t cut = max_len < 2048 ? 1 : std::max<int64_t>(1, std::min(full / wide, most));
  p.wide = cols >= 64 && wide * cut >= 384;
  p.waves = groups(16) <= 256 ? 8 : 4;
  int64_t n = p.wide ? cut : max_len < 2048 ? 1 : std::min(256 / groups(16), most);
  n = std::max<int64_t>(1, std::min<int64_t>(n, TREE_MAX_SPLIT));
  p.chunk = (int)std::min<int64_t>((((int64_t)max_len + n - 1) / n + 63) / 64 * 64, 1 << 30);
  p.n_split = (int)((max_len + (int64_t)p.chunk - 1) / p.chunk);
  return p;
}

hipError_t launch_kv8_tree(const int32_t* parent, const Kv8Rows& b, int words, uint64_t* mask, int32_t* pos, hipStream_t st) {
  if (b.rows <= 0 || b.n_seqs <= 0) return hipSuccess;
  return kv8_launch(k_kv8_tree, dim3(b.n_seqs), dim3(64), st, parent, b, words, mask, pos);
}

hipError_t launch_kv8_tree_attention(int dtype, const Kv8TreeAttn& t, hipStream_t st) {
  const Kv8Attn& a = t.a;
  if (a.b.rows <= 0 || a.b.n_seqs <= 0) return hipSuccess;
  if ((a.c.hd != 64 && a.c.hd != 128) || a.plan.n_split < 1 || a.plan.n_split > TREE_MAX_SPLIT || a.plan.chunk % 64 ||
      (a.plan.n_split > 1 && (!a.part_o || !a.part_ml)))
    return hipErrorInvalidValue;
  const bool w = a.c.hd == 128;
  hipError_t e;
  if (dtype == 1) e = w ? run<bf16_t, 128>(t, st) : run<bf16_t, 64>(t, st);
  else e = w ? run<float, 128>(t, st) : run<float, 64>(t, st);
  if (e != hipSuccess || a.plan.n_split == 1) return e;
  if (dtype == 1) return w ? merge<bf16_t, 128>(a, st) : merge<bf16_t, 64>(a, st);
  return w ? merge<float, 128>(a, st) : merge<float, 64>(a, st);
}

hipError_t launch_kv8_accept(const Kv8Pool& c, const Kv8Rows& b, const uint64_t* mask, int words, const int32_t* last,
                             int32_t* new_len, hipStream_t st) {
  if (b.n_seqs <= 0) return hipSuccess;
  if (c.hd != 64 && c.hd != 128) return hipErrorInvalidValue;
  const int64_t grid = (int64_t)b.n_seqs * c.n_kv * 2;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  const AcceptArgs a{c, b, mask, words, last, new_len};
  const dim3 g((unsigned)grid), t(64 * ACCEPT_WAVES);
  return c.hd == 128 ? kv8_launch(k_kv8_accept<128>, g, t, st, a) : kv8_launch(k_kv8_accept<64>, g, t, st, a);
}
