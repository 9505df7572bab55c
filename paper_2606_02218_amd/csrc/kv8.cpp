// C entry points of the rotary positions, the 8-bit key/value cache, drafted trees
// over it and sampling from given logits (include/rollout.h): argument checks, then
// the launchers.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>

#include "rollout.h"
#include "rg_kernels.h"

int rg_set_error(int code, const char* msg);

namespace {

int bad(const char* who, const char* what, int code = RG_EINVAL) {
  char msg[160];
  std::snprintf(msg, sizeof msg, "%s: %s", who, what);
  return rg_set_error(code, msg);
}

int launched(const char* who, hipError_t e) {
  return e == hipSuccess ? RG_OK : bad(who, hipGetErrorString(e), RG_EHIP);
}

bool aligned(const void* p) { return (uintptr_t)p % 16 == 0; }

// Whether two views of `rows` rows, hd elements of eb bytes a head, share an element.
// Where their ranges meet, as those of parts of one projection's output do, each
// pair of heads is compared over the rows; rows that do not go in step are taken to
// meet.  (More pairs of heads than any model has: not looked at.)
bool overlap(const HeadView& a, int a_heads, const HeadView& b, int b_heads, int rows, int hd, int eb) {
  auto range = [&](const HeadView& x, int heads, int64_t& lo, int64_t& hi) {
    const int64_t r = (rows - 1) * x.row, h = (heads - 1) * x.head;
    lo = (int64_t)x.p + eb * (std::min<int64_t>(r, 0) + std::min<int64_t>(h, 0));
    hi = (int64_t)x.p + eb * (std::max<int64_t>(r, 0) + std::max<int64_t>(h, 0) + hd);
  };
  int64_t al, ah, bl, bh;
  range(a, a_heads, al, ah);
  range(b, b_heads, bl, bh);
  if (ah <= bl || bh <= al) return false;
  if (rows > 1 && a.row != b.row) return true;
  if ((int64_t)a_heads * b_heads > 1 << 20) return false;
  const int64_t wide = (int64_t)hd * eb, step = rows > 1 ? std::abs(a.row) * eb : 0;
  for (int i = 0; i < a_heads; ++i)
    for (int j = 0; j < b_heads; ++j) {
      int64_t d = std::abs((int64_t)b.p + j * b.head * eb - (int64_t)a.p - i * a.head * eb);   // and rows apart: d - n * step
      if (step) {
        const int64_t n = std::min<int64_t>(d / step, rows - 1);
        d -= n * step;
        if (n + 1 < rows) d = std::min(d, step - d);
      }
      if (d < wide) return true;
    }
  return false;
}

// Every host check of a cache and a batch; fills the kernels' forms.
int cache_args(const char* who, const rg_kv8_cache* c, const rg_kv8_batch* b, int32_t dtype, Kv8Pool* pool,
               Kv8Rows* rows) {
  if (!c || !b) return bad(who, "NULL argument");
  if (dtype != RG_DTYPE_F32 && dtype != RG_DTYPE_BF16) return bad(who, "unknown dtype");
  if (!c->k || !c->v || !c->k_scale || !c->v_scale) return bad(who, "NULL cache pointer");
  if (!aligned(c->k) || !aligned(c->v)) return bad(who, "cache codes are not 16-byte aligned");
  if (c->pages < 1 || c->n_kv < 1) return bad(who, "pages and n_kv must be >= 1");
  if (c->head_dim != 64 && c->head_dim != 128) return bad(who, "head_dim must be 64 or 128", RG_EUNSUPPORTED);
  int shift = 0;
  while (shift < 6 && (16 << shift) < c->page_tokens) ++shift;
  if (c->page_tokens != 16 << shift)
    return bad(who, "page_tokens must be 16, 32, 64, .. 1024", RG_EUNSUPPORTED);
  if (c->pages > (INT32_MAX >> shift) / c->n_kv) return bad(who, "the cache has 2^31 blocks or more", RG_EUNSUPPORTED);
  if (b->rows < 0 || b->n_seqs < 0 || b->n_seqs > (1 << 28)) return bad(who, "rows or n_seqs out of range");
  if (b->rows > 0) {
    if (!b->page_tab || !b->seq_len) return bad(who, "NULL page_tab or seq_len");
    if (b->n_seqs < 1 || b->tab_rows < 1 || b->tab_stride < 1)
      return bad(who, "n_seqs, tab_rows and tab_stride must be >= 1");
    if (!b->seq_off && b->rows != b->n_seqs) return bad(who, "without seq_off, rows must equal n_seqs");
    if ((int64_t)b->tab_stride * c->page_tokens > (1 << 30)) return bad(who, "tab_stride * page_tokens exceeds 2^30");
  }
  *pool = Kv8Pool{(uint8_t*)c->k, (uint8_t*)c->v, c->k_scale, c->v_scale, (int)c->pages, c->n_kv, c->head_dim, shift};
  *rows = Kv8Rows{b->page_tab, b->tab_rows, b->tab_stride, b->tab_row, b->seq_off, b->seq_len, 0, b->n_seqs, b->rows,
                  nullptr};
  return RG_OK;
}

int rope_args(const char* who, const float* co, const float* si, int32_t n_pos, int32_t rot_dim, int32_t head_dim,
              int32_t layout, RopeTable* t) {
  if (layout != RG_ROPE_HALF && layout != RG_ROPE_INTERLEAVED) return bad(who, "unknown layout");
  if (rot_dim < 2 || rot_dim % 2 || rot_dim > head_dim) return bad(who, "rot_dim must be even and in [2, head_dim]");
  if (!co || !si) return bad(who, "NULL table");
  if (n_pos < 1) return bad(who, "n_pos < 1");
  *t = RopeTable{co, si, n_pos, rot_dim / 2, layout};
  return RG_OK;
}

// What the calls on drafted trees ask beyond cache_args: offsets, and a mask's width.
int tree_args(const char* who, const rg_kv8_batch* b, int32_t words) {
  if (words < 1 || words > RG_KV8_TREE_WORDS) return bad(who, "words must be in [1, 64]");
  if (b->rows > 0 && !b->seq_off) return bad(who, "NULL seq_off");
  return RG_OK;
}

// The sizes and settings of a sampling call.
DrawArgs draw_args(int32_t rows, int32_t vocab, const rg_sample_options& o) {
  DrawArgs a{};
  a.rows = rows;
  a.vocab = vocab;
  a.temperature = o.temperature;
  a.top_k = (int)std::min<int64_t>(o.top_k, INT32_MAX);
  a.top_p = o.top_p;
  a.min_p = o.min_p;
  a.temperature_rows = o.temperature_rows;
  a.top_k_rows = o.top_k_rows;
  a.top_p_rows = o.top_p_rows;
  a.min_p_rows = o.min_p_rows;
  return a;
}

}  // namespace

extern "C" {

int rg_rope_table(float* cos_tab, float* sin_tab, int32_t n_pos, int32_t rot_dim, double theta, int32_t scaling,
                  double factor, double length, double slow, double fast, void* stream) {
  const char* who = "rg_rope_table";
  if (!cos_tab || !sin_tab) return bad(who, "NULL argument");
  if (n_pos < 1 || rot_dim < 2 || rot_dim % 2) return bad(who, "n_pos < 1, or rot_dim odd or < 2");
  if (!(theta > 0.0) || !std::isfinite(theta)) return bad(who, "theta must be > 0");
  if (scaling < RG_ROPE_PLAIN || scaling > RG_ROPE_BANDS) return bad(who, "unknown scaling");
  if (scaling != RG_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return bad(who, "factor must be >= 1");
  if (scaling == RG_ROPE_BASE && rot_dim < 4) return bad(who, "a raised base needs rot_dim >= 4");
  if (scaling == RG_ROPE_BANDS &&
      (!(length > 0.0) || !std::isfinite(length) || !(slow < fast) || !std::isfinite(slow) || !std::isfinite(fast)))
    return bad(who, "bands need length > 0 and slow < fast");
  return launched(who, launch_rope_table(cos_tab, sin_tab, n_pos,
                                         RopeFreqs{rot_dim / 2, scaling, theta, factor, length, slow, fast},
                                         (hipStream_t)stream));
}

int rg_rope(int32_t dtype, const void* x, int64_t x_row, int64_t x_head, void* y, int64_t y_row, int64_t y_head,
            const int32_t* pos, int32_t rows, int32_t heads, int32_t head_dim, const float* cos_tab,
            const float* sin_tab, int32_t n_pos, int32_t rot_dim, int32_t layout, int32_t inverse, void* stream) {
  const char* who = "rg_rope";
  if (dtype != RG_DTYPE_F32 && dtype != RG_DTYPE_BF16) return bad(who, "unknown dtype");
  if (rows < 0 || heads < 0 || head_dim < 2 || head_dim % 2) return bad(who, "negative sizes, or head_dim odd or < 2");
  RopeTable t;
  int rc = rope_args(who, cos_tab, sin_tab, n_pos, rot_dim, head_dim, layout, &t);
  if (rc) return rc;
  if (rows == 0 || heads == 0) return RG_OK;
  if (!x || !y || !pos) return bad(who, "NULL argument");
  if (x == y && (x_row != y_row || x_head != y_head)) return bad(who, "y overlaps x with other strides");
  return launched(who, launch_rope(dtype, HeadView{x, x_row, x_head}, HeadOut{y, y_row, y_head}, pos, rows, heads,
                                   head_dim, t, inverse != 0, (hipStream_t)stream));
}

int rg_kv8_append(const rg_kv8_cache* cache, const rg_kv8_batch* batch, int32_t dtype, const void* k, int64_t k_row,
                  int64_t k_head, const void* v, int64_t v_row, int64_t v_head, const void* q, int64_t q_row,
                  int64_t q_head, void* q_out, int64_t qo_row, int64_t qo_head, int32_t n_q, const float* cos_tab,
                  const float* sin_tab, int32_t n_pos, int32_t rot_dim, int32_t layout, void* stream) {
  const char* who = "rg_kv8_append";
  Kv8Pool pool;
  Kv8Rows rows;
  int rc = cache_args(who, cache, batch, dtype, &pool, &rows);
  if (rc) return rc;
  RopeTable t{nullptr, nullptr, 0, 0, RG_ROPE_HALF};
  if (rot_dim != 0 && (rc = rope_args(who, cos_tab, sin_tab, n_pos, rot_dim, pool.hd, layout, &t))) return rc;
  if (q && (n_q < 1 || n_q % pool.n_kv)) return bad(who, "n_q must be a multiple of n_kv");
  if (rows.rows == 0) return RG_OK;
  if (!k || !v) return bad(who, "NULL k or v");
  if (q && !q_out) return bad(who, "NULL q_out");
  if (q && q == q_out && (q_row != qo_row || q_head != qo_head)) return bad(who, "q_out overlaps q with other strides");
  if (q) {   // keys, values and queries are taken by different waves, in any order
    const int eb = dtype == RG_DTYPE_BF16 ? 2 : 4, n = rows.rows;
    const HeadView o{q_out, qo_row, qo_head};
    if (overlap(o, n_q, HeadView{k, k_row, k_head}, pool.n_kv, n, pool.hd, eb) ||
        overlap(o, n_q, HeadView{v, v_row, v_head}, pool.n_kv, n, pool.hd, eb))
      return bad(who, "q_out overlaps k or v");
    if (q != q_out && overlap(o, n_q, HeadView{q, q_row, q_head}, n_q, n, pool.hd, eb))
      return bad(who, "q_out overlaps q without being q");
  }
  return launched(who, launch_kv8_append(dtype, pool, rows, HeadView{k, k_row, k_head}, HeadView{v, v_row, v_head},
                                         HeadView{q, q_row, q_head}, HeadOut{q_out, qo_row, qo_head}, n_q, t,
                                         (hipStream_t)stream));
}

int64_t rg_kv8_attention_scratch(int32_t n_q, int32_t n_kv, int32_t head_dim, int32_t rows, int32_t n_seqs,
                                 int32_t has_off, int32_t max_len) {
  if (n_q < 1 || n_kv < 1 || n_q % n_kv || head_dim < 1 || rows < 0 || n_seqs < 0 || max_len < 1)
    return bad("rg_kv8_attention_scratch", "bad sizes");
  if (rows == 0 || n_seqs == 0) return 0;
  const Kv8Plan p = kv8_plan(rows, n_seqs, has_off != 0, true, n_q, n_kv, max_len, INT32_MAX);
  return 4 * kv8_part_floats(rows, p, n_q, head_dim);
}

int rg_kv8_attention(const rg_kv8_cache* cache, const rg_kv8_batch* batch, int32_t dtype, const void* q,
                     int64_t q_row, int64_t q_head, int32_t n_q, void* out, float scale, int32_t max_len,
                     void* scratch, int64_t scratch_bytes, void* stream) {
  const char* who = "rg_kv8_attention";
  Kv8Attn a{};
  int rc = cache_args(who, cache, batch, dtype, &a.c, &a.b);
  if (rc) return rc;
  if (n_q < 1 || n_q % a.c.n_kv) return bad(who, "n_q must be a multiple of n_kv");
  if (n_q / a.c.n_kv > 128) return bad(who, "more than 128 query heads per kv head", RG_EUNSUPPORTED);
  // scores are taken in base 2: 0 times an infinite factor would be NaN
  if (!(scale > 0.f) || !std::isfinite(scale * 1.44269504f)) return bad(who, "scale must be > 0 and at most 2.3e38");
  if (max_len < 1) return bad(who, "max_len < 1");
  if (a.b.rows == 0) return RG_OK;
  if (!q || !out) return bad(who, "NULL q or out");
  if (!aligned(out) || !aligned(scratch)) return bad(who, "out or scratch is not 16-byte aligned");
  a.q = HeadView{q, q_row, q_head};
  a.out = out;
  a.n_q = n_q;
  a.scale = scale;
  a.plan = kv8_plan(a.b.rows, a.b.n_seqs, a.b.seq_off != nullptr, true, n_q, a.c.n_kv, max_len, INT32_MAX);
  a.part_o = (float*)scratch;
  a.part_ml = a.part_o ? a.part_o + (int64_t)a.b.rows * a.plan.n_split * n_q * a.c.hd : nullptr;
  const int64_t need = 4 * kv8_part_floats(a.b.rows, a.plan, n_q, a.c.hd);
  if (need > 0 && (!scratch || scratch_bytes < need)) return bad(who, "scratch is smaller than rg_kv8_attention_scratch()");
  if ((rc = launched(who, launch_kv8_attention(dtype, false, a, (hipStream_t)stream)))) return rc;
  return launched(who, launch_kv8_merge(dtype, false, a, (hipStream_t)stream));
}

int rg_kv8_tree(const int32_t* parent, const int32_t* seq_off, const int32_t* seq_len, int32_t n_seqs, int32_t rows,
                int32_t words, uint64_t* mask, int32_t* pos, void* stream) {
  const char* who = "rg_kv8_tree";
  if (rows < 0 || n_seqs < 0 || n_seqs > (1 << 24)) return bad(who, "rows or n_seqs out of range");
  if (words < 1 || words > RG_KV8_TREE_WORDS) return bad(who, "words must be in [1, 64]");
  if (rows == 0 || n_seqs == 0) return RG_OK;
  if (!parent || !seq_off || !seq_len || !mask || !pos) return bad(who, "NULL argument");
  const Kv8Rows b{nullptr, 0, 0, nullptr, seq_off, seq_len, 0, n_seqs, rows, nullptr};
  return launched(who, launch_kv8_tree(parent, b, words, mask, pos, (hipStream_t)stream));
}

int64_t rg_kv8_tree_attention_scratch(int32_t dtype, int32_t n_q, int32_t n_kv, int32_t head_dim, int32_t rows, int32_t n_seqs,
                                      int32_t words, int32_t max_len) {
  if ((dtype != RG_DTYPE_F32 && dtype != RG_DTYPE_BF16) || n_q < 1 || n_kv < 1 || n_q % n_kv || n_q / n_kv > 128 ||
      head_dim < 1 || rows < 0 || n_seqs < 0 || max_len < 1 || words < 1 || words > RG_KV8_TREE_WORDS)
    return bad("rg_kv8_tree_attention_scratch", "bad sizes");
  if (rows == 0 || n_seqs == 0) return 0;
  return 4 * kv8_tree_part_floats(rows, kv8_tree_plan(dtype, rows, n_seqs, n_q, n_kv, max_len), n_q, head_dim);
}

int rg_kv8_tree_attention(const rg_kv8_cache* cache, const rg_kv8_batch* batch, int32_t dtype, const void* q, int64_t q_row,
                          int64_t q_head, int32_t n_q, const uint64_t* mask, int32_t words, void* out, float scale,
                          int32_t max_len, void* scratch, int64_t scratch_bytes, void* stream) {
  const char* who = "rg_kv8_tree_attention";
  Kv8TreeAttn t{};
  Kv8Attn& a = t.a;
  int rc = cache_args(who, cache, batch, dtype, &a.c, &a.b);
  if (rc || (rc = tree_args(who, batch, words))) return rc;
  if (n_q < 1 || n_q % a.c.n_kv) return bad(who, "n_q must be a multiple of n_kv");
  if (n_q / a.c.n_kv > 128) return bad(who, "more than 128 query heads per kv head", RG_EUNSUPPORTED);
  if (!(scale > 0.f) || !std::isfinite(scale * 1.44269504f)) return bad(who, "scale must be > 0 and at most 2.3e38");
  if (max_len < 1) return bad(who, "max_len < 1");
  if (a.b.rows == 0) return RG_OK;
  if (!q || !out || !mask) return bad(who, "NULL q, out or mask");
  if (!aligned(out) || !aligned(scratch)) return bad(who, "out or scratch is not 16-byte aligned");
  a.q = HeadView{q, q_row, q_head};
  a.out = out;
  a.mask = mask;
  a.words = words;
  a.n_q = n_q;
  a.scale = scale;
  const Kv8TreePlan plan = kv8_tree_plan(dtype, a.b.rows, a.b.n_seqs, n_q, a.c.n_kv, max_len);
  t.wide = plan.wide;
  a.plan.waves = plan.waves;
  a.plan.n_split = plan.n_split;
  a.plan.chunk = plan.chunk;
  const int64_t need = 4 * kv8_tree_part_floats(a.b.rows, plan, n_q, a.c.hd);
  if (need > 0 && (!scratch || scratch_bytes < need))
    return bad(who, "scratch is smaller than rg_kv8_tree_attention_scratch()");
  a.part_o = (float*)scratch;
  a.part_ml = a.part_o ? a.part_o + (int64_t)a.b.rows * a.plan.n_split * n_q * a.c.hd : nullptr;
  return launched(who, launch_kv8_tree_attention(dtype, t, (hipStream_t)stream));
}

int rg_kv8_accept(const rg_kv8_cache* cache, const rg_kv8_batch* batch, const uint64_t* mask, int32_t words,
                  const int32_t* last, int32_t* new_len, void* stream) {
  const char* who = "rg_kv8_accept";
  Kv8Pool pool;
  Kv8Rows rows;
  int rc = cache_args(who, cache, batch, RG_DTYPE_BF16, &pool, &rows);
  if (rc || (rc = tree_args(who, batch, words))) return rc;
  if (rows.n_seqs == 0) return RG_OK;
  if (!batch->seq_off || !batch->seq_len || !new_len) return bad(who, "NULL seq_off, seq_len or new_len");
  if (rows.rows > 0 && (!mask || !last)) return bad(who, "NULL mask or last");
  // read by workgroups of the sequence that writes it, and of others
  auto meets = [&](const void* p, int64_t bytes) {
    return p && (const char*)p < (const char*)(new_len + rows.n_seqs) && (const char*)new_len < (const char*)p + bytes;
  };
  const int64_t n = rows.n_seqs, blocks = (int64_t)pool.pages * pool.n_kv << pool.sub_shift, codes = blocks * 16 * pool.hd;
  if (meets(batch->seq_len, 4 * n) || meets(last, 4 * n) || meets(batch->seq_off, 4 * (n + 1)) || meets(batch->tab_row, 4 * n) ||
      meets(batch->page_tab, 4 * (int64_t)batch->tab_rows * batch->tab_stride) || meets(mask, 8 * (int64_t)rows.rows * words) ||
      meets(pool.k, codes) || meets(pool.v, codes) || meets(pool.k_scale, 4 * blocks) || meets(pool.v_scale, 4 * blocks))
    return bad(who, "new_len overlaps what the call reads");
  return launched(who, launch_kv8_accept(pool, rows, mask, words, last, new_len, (hipStream_t)stream));
}

int64_t rg_sample_scratch(int32_t rows, int32_t vocab, const rg_sample_options* options) {
  const char* who = "rg_sample_scratch";
  if (!options) return bad(who, "NULL argument");
  if (rows < 0 || vocab < 1 || vocab > DRAW_MAX_VOCAB) return bad(who, "rows < 0, or vocab not in [1, 2^20]");
  return rows == 0 ? 0 : draw_scratch_bytes(draw_args(rows, vocab, *options));
}

int rg_sample(int32_t dtype, const void* logits, int64_t logits_row, int32_t rows, int32_t vocab, int32_t u_dtype, const void* u,
              const rg_sample_options* options, int32_t* tokens, float* logprobs, float* kept_logprobs, void* scratch,
              int64_t scratch_bytes, void* stream) {
  const char* who = "rg_sample";
  if (!options) return bad(who, "NULL argument");
  if (dtype != RG_DTYPE_F32 && dtype != RG_DTYPE_BF16) return bad(who, "unknown dtype");
  if (u_dtype != RG_DTYPE_F32 && u_dtype != RG_DTYPE_F64) return bad(who, "u must be fp32 or fp64");
  if (rows < 0 || vocab < 1) return bad(who, "rows < 0 or vocab < 1");
  if (vocab > DRAW_MAX_VOCAB) return bad(who, "vocab exceeds 2^20", RG_EUNSUPPORTED);
  const rg_sample_options& o = *options;
  if (!o.temperature_rows && !(o.temperature >= 0.0 && std::isfinite(o.temperature))) return bad(who, "temperature must be >= 0");
  if (!o.top_k_rows && o.top_k < 0) return bad(who, "top_k must be >= 0");
  if (!o.top_p_rows && !(o.top_p > 0.0 && o.top_p <= 1.0)) return bad(who, "top_p must be in (0, 1]");
  if (!o.min_p_rows && !(o.min_p >= 0.0 && o.min_p <= 1.0)) return bad(who, "min_p must be in [0, 1]");
  if (rows == 0) return RG_OK;
  if (!logits || !u || !tokens || !logprobs || !kept_logprobs) return bad(who, "NULL argument");
  DrawArgs a = draw_args(rows, vocab, o);
  if (!scratch || scratch_bytes < draw_scratch_bytes(a)) return bad(who, "scratch is smaller than rg_sample_scratch()");
  if (!aligned(scratch)) return bad(who, "scratch is not 16-byte aligned");
  a.logits = logits;
  a.row = logits_row;
  a.dtype = dtype;
  a.u = u;
  a.u64 = u_dtype == RG_DTYPE_F64;
  a.token = tokens;
  a.logprob = logprobs;
  a.kept = kept_logprobs;
  return launched(who, launch_draw(a, scratch, (hipStream_t)stream));
}

}  // extern "C"
