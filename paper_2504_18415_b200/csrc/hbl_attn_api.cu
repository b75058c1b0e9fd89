// extern "C" entry points from q, k, v to the input of W_o: rotary positions, the paged cache of attention states,
// attention over it.  Argument validation and dispatch; no device memory is allocated here.
#include <math.h>

#include "hbl_kv_cache.cuh"

using namespace hbl;

namespace {

constexpr int kMaxRotDim = 256;
constexpr int kMaxHeads = 1 << 20;      // rows of a call (token times head) and what the host computes of them stay in range

// A [tokens, heads, dim] tensor with strides: every piece of 8 elements has to lie on a 16-byte boundary.
int check_strided(const void* p, long long token_stride, long long head_stride) {
  if (!aligned(p, 16)) return HBL_ERR_ALIGN;
  if (token_stride % 8 != 0 || head_stride % 8 != 0) return HBL_ERR_ALIGN;
  if (token_stride < 0 || head_stride < 0) return HBL_ERR_SHAPE;
  return HBL_OK;
}
// One that is written: two of its heads may not lie on each other, because different thread blocks write them.  Where neither
// all heads of a token lie between one token and the next nor the other way round, head h of token t may lie on head h - i of
// token t + j; so it does where i head strides and j token strides differ by less than a head.
bool heads_overlap(long long token_stride, long long head_stride, long long tokens, long long heads, long long head_dim) {
  using wide = __int128;                                        // strides are the caller's: products may pass 64 bits
  if (tokens <= 1) return heads > 1 && head_stride < head_dim;
  if (heads <= 1) return token_stride < head_dim;
  if (token_stride < head_dim || head_stride < head_dim) return true;
  if (token_stride >= (wide)(heads - 1) * head_stride + head_dim || head_stride >= (wide)(tokens - 1) * token_stride + head_dim) return false;
  const bool by_head = heads <= tokens;                         // along the shorter axis, the nearest two of the other's
  const long long n = by_head ? heads : tokens, m = by_head ? tokens : heads;
  const long long step = by_head ? head_stride : token_stride, other = by_head ? token_stride : head_stride;
  for (long long i = 1; i < n; ++i) {
    const wide at = (wide)i * step, j = at / other;
    if (j >= 1 && j < m && at - j * other < head_dim) return true;
    if (j + 1 < m && (j + 1) * other - at < head_dim) return true;
    if (j >= m) return false;                                   // beyond the last of them, and so is all that follows
  }
  return false;
}
int check_written(const void* p, long long token_stride, long long head_stride, int tokens, int heads, int head_dim) {
  const int rc = check_strided(p, token_stride, head_stride);
  if (rc != HBL_OK) return rc;
  return heads_overlap(token_stride, head_stride, tokens, heads, head_dim) ? HBL_ERR_SHAPE : HBL_OK;
}
int check_rotation(const float* table, int n_pos, int rot_dim, int head_dim, int layout) {
  if (layout != HBL_ROPE_HALF && layout != HBL_ROPE_INTERLEAVED) return HBL_ERR_FORMAT;
  if (rot_dim < 16 || rot_dim % 16 != 0 || rot_dim > head_dim || n_pos <= 0) return HBL_ERR_SHAPE;
  return aligned(table, 16) ? HBL_OK : HBL_ERR_ALIGN;
}

int check_cache(const hbl_kv_cache_t* c, KvView* v) {
  if (!c) return HBL_ERR_NULL;
  if (c->bits != 3 && c->bits != 4 && c->bits != 8 && c->bits != 16) return HBL_ERR_BITS;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return HBL_ERR_SHAPE;
  if (c->n_kv_heads <= 0 || c->n_pages <= 0) return HBL_ERR_SHAPE;
  if (c->page_size < 16 || c->page_size > 4096 || !is_pow2(c->page_size)) return HBL_ERR_SHAPE;
  if ((long long)c->n_pages * c->n_kv_heads * c->page_size > 0x7fffffffLL) return HBL_ERR_TOO_LARGE;   // row numbers: 32 bits
  if (!c->k || !c->v) return HBL_ERR_NULL;
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return HBL_ERR_ALIGN;
  if (c->bits == 16) {
    if (c->k_scale || c->v_scale) return HBL_ERR_FORMAT;
  } else {
    if (!c->k_scale || !c->v_scale) return HBL_ERR_NULL;
    if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return HBL_ERR_ALIGN;
  }
  if (c->bos_k || c->bos_v || c->bos_k_scale || c->bos_v_scale) {
    if (c->bits >= 8) return HBL_ERR_BITS;                       // (at 8 bits and more there is nothing to keep better)
    if (!c->bos_k || !c->bos_v || !c->bos_k_scale || !c->bos_v_scale) return HBL_ERR_NULL;
    if (!aligned(c->bos_k, 16) || !aligned(c->bos_v, 16) || !aligned(c->bos_k_scale, 4) || !aligned(c->bos_v_scale, 4))
      return HBL_ERR_ALIGN;
    if (c->n_slots <= 0) return HBL_ERR_SHAPE;
  }
  v->k = static_cast<unsigned char*>(c->k);
  v->v = static_cast<unsigned char*>(c->v);
  v->k_scale = c->k_scale;
  v->v_scale = c->v_scale;
  v->bos_k = static_cast<unsigned char*>(c->bos_k);
  v->bos_v = static_cast<unsigned char*>(c->bos_v);
  v->bos_k_scale = c->bos_k_scale;
  v->bos_v_scale = c->bos_v_scale;
  v->n_pages = c->n_pages;
  v->page_shift = ilog2(c->page_size);
  v->n_kv_heads = c->n_kv_heads;
  v->head_dim = c->head_dim;
  v->bits = c->bits;
  v->n_slots = c->n_slots;
  return HBL_OK;
}
int check_batch(const hbl_kv_batch_t* b, BatchView* v) {
  if (!b) return HBL_ERR_NULL;
  if (b->n_seqs < 0 || b->tokens < 0 || b->max_pages < 0 || b->max_q_len < 0 || b->max_kv_len < 0) return HBL_ERR_SHAPE;
  if (b->max_kv_len > kMaxKvLen) return HBL_ERR_TOO_LARGE;
  *v = {b->q_start, b->kv_len, b->pages, b->bos_slot, b->n_seqs, b->tokens, b->max_pages,
        b->max_q_len < b->tokens ? b->max_q_len : b->tokens, b->max_kv_len};
  if (b->n_seqs == 0 || b->tokens == 0) return HBL_OK;            // nothing will be looked at
  if (!b->q_start || !b->kv_len || !b->pages) return HBL_ERR_NULL;
  if (!aligned(b->q_start, 4) || !aligned(b->kv_len, 4) || !aligned(b->pages, 4) || !aligned(b->bos_slot, 4)) return HBL_ERR_ALIGN;
  return HBL_OK;
}
bool nothing(const BatchView& b) { return b.n_seqs == 0 || b.tokens == 0; }

// How a call is made: sequences of up to `few` query rows on the streaming kernel, longer ones on the tensor-core
// tiles; a single sequence, whose length the bound says, on one of them alone.  The streaming kernel reads
// the keys once for 16 rows, so its time goes up in steps (8192 tokens, heads of 128, us at 8, 16, 32 rows: streaming / tiles):
//                                3 bits                    4 bits                    8 bits                    16 bits
//   1 sequence, 32 key heads     32 46  62 /  73  73  73   30 46  58 /  69  70  71   38 54  73 /  75  75  79   48 56  87 /  52  52  52
//   32 sequences, 8 key heads   101 183 305 / 430 429 430  103 171 276 / 376 376 377  148 228 437 / 409 412 417  208 267 364 / 257 255 256
// Up to 16 rows streaming wins over codes by far and loses at 16 bits by 8 % and 5 % from 9 rows on.  At 3 and 4 bits it still
// wins at 32 rows (not at 48: 97 and 385 us, 93 and 344), at 8 bits the two meet there: the border there could be later.
constexpr int kFewRows = 16;
struct AttnCall {
  bool use_rows, use_tiles;
  int few_rows, few_tiles;             // the border as each kernel sees it
  AttnPlan rows, tiles;
  size_t rows_lse, tiles_o, tiles_lse, workspace;     // byte offsets of the parts (rows_o at 0), and the bytes of all
};
AttnCall plan_attention(const KvView& c, const BatchView& b, int n_heads) {
  AttnCall w{};
  const int group = n_heads / c.n_kv_heads;
  w.use_tiles = (long)b.max_q_len * group > kFewRows;
  w.use_rows = !w.use_tiles || b.n_seqs > 1;
  w.few_rows = kFewRows;
  w.few_tiles = w.use_rows ? kFewRows : 0;
  w.rows.splits = w.tiles.splits = 1;
  if (w.use_rows) w.rows = plan_attention_rows(c, b, n_heads, w.few_rows);
  if (w.use_tiles) w.tiles = plan_attention_tiles(c, b, n_heads, w.few_tiles);
  size_t off = 0;
  auto take = [&](size_t& at, size_t floats) { at = off; off = align_up(off + floats * sizeof(float), 1024); };
  if (w.rows.splits > 1) {
    const size_t rows = (size_t)w.rows.splits * b.n_seqs * c.n_kv_heads * w.rows.cap;
    size_t rows_o;
    take(rows_o, rows * c.head_dim);
    take(w.rows_lse, rows);
  }
  if (w.tiles.splits > 1) {
    const size_t rows = (size_t)w.tiles.splits * b.tokens * n_heads;
    take(w.tiles_o, rows * c.head_dim);
    take(w.tiles_lse, rows);
  }
  w.workspace = off;
  return w;
}

}  // namespace

extern "C" {

int hbl_rope_frequencies(double base, int rot_dim, int scaling, double factor, double trained_len, double slow, double fast,
                         double* freq_out) {
  if (!freq_out) return HBL_ERR_NULL;
  if (rot_dim < 2 || rot_dim > kMaxRotDim || rot_dim % 2 != 0) return HBL_ERR_SHAPE;
  if (scaling < HBL_ROPE_PLAIN || scaling > HBL_ROPE_PARTS) return HBL_ERR_FORMAT;
  if (!(base > 1.0) || !isfinite(base)) return HBL_ERR_SHAPE;
  if (scaling != HBL_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return HBL_ERR_SHAPE;
  if (scaling == HBL_ROPE_BASE && rot_dim < 4) return HBL_ERR_SHAPE;
  if (scaling == HBL_ROPE_PARTS && (!(trained_len > 0.0) || !isfinite(trained_len) || !(slow > 0.0) || !(fast > slow) || !isfinite(fast)))
    return HBL_ERR_SHAPE;
  if (scaling == HBL_ROPE_BASE) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / rot_dim);
    if (scaling == HBL_ROPE_LINEAR) f /= factor;
    if (scaling == HBL_ROPE_PARTS) {
      const double turns = trained_len * f / (2.0 * 3.14159265358979323846);
      const double keep = turns >= fast ? 1.0 : turns <= slow ? 0.0 : (turns - slow) / (fast - slow);
      f = keep * f + (1.0 - keep) * (f / factor);
    }
    freq_out[i] = f;
  }
  return HBL_OK;
}

int hbl_rope_table(const double* freq, int n_freq, double amplitude, int first_pos, int n_pos, float* table, void* stream) {
  if (n_freq <= 0 || n_freq > kMaxRotDim / 2 || n_pos < 0 || first_pos < 0) return HBL_ERR_SHAPE;
  if ((long long)first_pos + n_pos > 0x7fffffffLL) return HBL_ERR_TOO_LARGE;
  if (!isfinite(amplitude)) return HBL_ERR_SHAPE;
  if (n_pos == 0) return HBL_OK;
  if (!freq || !table) return HBL_ERR_NULL;
  if (!aligned(table, 16)) return HBL_ERR_ALIGN;
  return launch_rope_table(freq, n_freq, amplitude, first_pos, n_pos, table, static_cast<cudaStream_t>(stream));
}

int hbl_rope(const hbl_rope_t* a, void* stream) {
  if (!a) return HBL_ERR_NULL;
  if (a->dtype != HBL_F32 && a->dtype != HBL_BF16) return HBL_ERR_FORMAT;
  if (a->tokens < 0 || a->n_heads <= 0 || a->head_dim < 8 || a->head_dim > kMaxRotDim || a->head_dim % 8 != 0) return HBL_ERR_SHAPE;
  int rc = check_rotation(a->table, a->n_pos, a->rot_dim, a->head_dim, a->layout);
  if (rc != HBL_OK) return rc;
  if (a->tokens == 0) return HBL_OK;
  if (!a->x || !a->positions || !a->table || !a->out) return HBL_ERR_NULL;
  if ((rc = check_strided(a->x, a->x_token_stride, a->x_head_stride)) != HBL_OK) return rc;
  if ((rc = check_written(a->out, a->out_token_stride, a->out_head_stride, a->tokens, a->n_heads, a->head_dim)) != HBL_OK) return rc;
  if (a->x == a->out && (a->x_token_stride != a->out_token_stride || a->x_head_stride != a->out_head_stride)) return HBL_ERR_SHAPE;
  if (!aligned(a->positions, 4)) return HBL_ERR_ALIGN;
  return launch_rope(a->x, a->dtype, a->tokens, a->n_heads, a->head_dim, a->x_token_stride, a->x_head_stride, a->positions, a->table,
                     a->n_pos, a->rot_dim, a->layout, a->backward != 0, a->out, a->out_token_stride, a->out_head_stride,
                     static_cast<cudaStream_t>(stream));
}

int hbl_kv_append(const hbl_kv_cache_t* cache, const hbl_kv_batch_t* batch, const hbl_kv_append_t* a, void* stream) {
  KvView c{};
  BatchView b{};
  int rc = check_cache(cache, &c);
  if (rc != HBL_OK) return rc;
  if ((rc = check_batch(batch, &b)) != HBL_OK) return rc;
  if (!a) return HBL_ERR_NULL;
  if (c.bits != 16 && (!(a->eps > 0.0f) || !isfinite(a->eps))) return HBL_ERR_EPS;
  if (a->table && (rc = check_rotation(a->table, a->n_pos, a->rot_dim, c.head_dim, a->layout)) != HBL_OK) return rc;
  if (a->q && a->n_heads <= 0) return HBL_ERR_SHAPE;
  if (nothing(b)) return HBL_OK;
  if (!a->k || !a->v) return HBL_ERR_NULL;
  if ((a->q != nullptr) != (a->q_out != nullptr) || (a->q && !a->table)) return HBL_ERR_NULL;
  if ((rc = check_strided(a->k, a->k_token_stride, a->k_head_stride)) != HBL_OK) return rc;
  if ((rc = check_strided(a->v, a->v_token_stride, a->v_head_stride)) != HBL_OK) return rc;
  if (a->q) {
    if ((rc = check_strided(a->q, a->q_token_stride, a->q_head_stride)) != HBL_OK) return rc;
    if ((rc = check_written(a->q_out, a->q_out_token_stride, a->q_out_head_stride, b.tokens, a->n_heads, c.head_dim)) != HBL_OK) return rc;
    if (a->q == a->q_out && (a->q_token_stride != a->q_out_token_stride || a->q_head_stride != a->q_out_head_stride)) return HBL_ERR_SHAPE;
  }
  if (!aligned(a->positions, 4)) return HBL_ERR_ALIGN;
  return launch_kv_append(c, b, *a, static_cast<cudaStream_t>(stream));
}

int hbl_kv_read(const hbl_kv_cache_t* cache, const hbl_kv_batch_t* batch, void* k_out, void* v_out, void* stream) {
  KvView c{};
  BatchView b{};
  int rc = check_cache(cache, &c);
  if (rc != HBL_OK) return rc;
  if ((rc = check_batch(batch, &b)) != HBL_OK) return rc;
  if (nothing(b)) return HBL_OK;
  if (!k_out || !v_out) return HBL_ERR_NULL;
  if (!aligned(k_out, 16) || !aligned(v_out, 16)) return HBL_ERR_ALIGN;
  return launch_kv_read(c, b, k_out, v_out, static_cast<cudaStream_t>(stream));
}

size_t hbl_attention_workspace_bytes(const hbl_kv_cache_t* cache, const hbl_kv_batch_t* batch, int n_heads) {
  KvView c{};
  BatchView b{};
  if (check_cache(cache, &c) != HBL_OK || check_batch(batch, &b) != HBL_OK || nothing(b)) return 0;
  if (n_heads <= 0 || n_heads > kMaxHeads || n_heads % c.n_kv_heads != 0) return 0;
  return plan_attention(c, b, n_heads).workspace;
}

int hbl_attention(const hbl_kv_cache_t* cache, const hbl_kv_batch_t* batch, const hbl_attention_t* args, void* workspace,
                  size_t workspace_bytes, void* stream) {
  KvView c{};
  BatchView b{};
  int rc = check_cache(cache, &c);
  if (rc != HBL_OK) return rc;
  if ((rc = check_batch(batch, &b)) != HBL_OK) return rc;
  if (!args) return HBL_ERR_NULL;
  if (args->n_heads <= 0 || args->n_heads % c.n_kv_heads != 0) return HBL_ERR_SHAPE;
  if (args->n_heads > kMaxHeads) return HBL_ERR_TOO_LARGE;
  if (!isfinite(args->sm_scale)) return HBL_ERR_SHAPE;
  if (nothing(b) || b.max_q_len == 0) return HBL_OK;
  if (!args->q || !args->out) return HBL_ERR_NULL;
  if ((rc = check_strided(args->q, args->q_token_stride, args->q_head_stride)) != HBL_OK) return rc;
  if ((rc = check_written(args->out, args->out_token_stride, args->out_head_stride, b.tokens, args->n_heads, c.head_dim)) != HBL_OK) return rc;
  if (!aligned(args->lse, 4)) return HBL_ERR_ALIGN;
  const AttnCall w = plan_attention(c, b, args->n_heads);
  if (w.workspace > 0 && !workspace) return HBL_ERR_NULL;
  if (!aligned(workspace, 1024)) return HBL_ERR_ALIGN;
  if (workspace_bytes < w.workspace) return HBL_ERR_WORKSPACE;
  AttnArgs a{};
  a.q = static_cast<const __nv_bfloat16*>(args->q);
  a.out = static_cast<__nv_bfloat16*>(args->out);
  a.lse = args->lse;
  a.q_ts = args->q_token_stride; a.q_hs = args->q_head_stride;
  a.o_ts = args->out_token_stride; a.o_hs = args->out_head_stride;
  a.n_heads = args->n_heads;
  a.group = args->n_heads / c.n_kv_heads;
  a.causal = args->causal != 0;
  a.scale_log2 = args->sm_scale * 1.4426950408889634f;
  char* ws = static_cast<char*>(workspace);
  const AttnParts parts = {reinterpret_cast<float*>(ws), reinterpret_cast<float*>(ws + w.rows_lse), reinterpret_cast<float*>(ws + w.tiles_o),
                           reinterpret_cast<float*>(ws + w.tiles_lse)};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (w.use_tiles && (rc = launch_attention_tiles(c, b, a, w.tiles, w.few_tiles, parts, s)) != HBL_OK) return rc;
  if (w.use_rows && (rc = launch_attention_rows(c, b, a, w.rows, w.few_rows, parts, w.use_tiles, s)) != HBL_OK) return rc;
  if (w.workspace > 0) return launch_attention_combine(c, b, a, w.rows, w.tiles, w.few_tiles, parts, s);
  return HBL_OK;
}

}  // extern "C"
