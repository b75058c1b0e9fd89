// Device-side view of the paged cache of attention states and of a batch of sequences over it (hbl.h:
// hbl_kv_cache_t, hbl_kv_batch_t), shared by the append, read and attention kernels.
#pragma once

#include "hbl_common.cuh"

namespace hbl {

struct KvView {
  unsigned char *k, *v;
  float *k_scale, *v_scale;
  unsigned char *bos_k, *bos_v;        // NULL: no 8-bit first token
  float *bos_k_scale, *bos_v_scale;
  int n_pages, page_shift, n_kv_heads, head_dim, bits, n_slots;
};
struct BatchView {
  const int32_t *q_start, *kv_len, *pages, *bos_slot;
  int n_seqs, tokens, max_pages, max_q_len, max_kv_len;
};

// The sequence of token t: the number of entries q_start[1..n_seqs] that are <= t (n_seqs: behind the last one).
// The whole warp searches for the same t, 32 entries a step.
__device__ __forceinline__ int find_sequence(const int32_t* __restrict__ q_start, int n_seqs, int t, int lane) {
  int lo = 0, n = n_seqs;                                     // the answer lies in [lo, lo + n]
  while (n > 0) {
    const int step = (n + 31) / 32;
    const int i = lo + (lane + 1) * step;                     // entry i counts when i <= lo + n
    const bool below = i <= lo + n && __ldg(q_start + i) <= t;
    const int full = __popc(__ballot_sync(0xffffffffu, below));
    const int hi = lo + n;
    lo += full * step;
    if (step == 1) break;
    n = min(step - 1, hi - lo);
  }
  return lo;
}

// Row number of (page, head, slot) in 64 bits: a long cache has more than 2^31 elements.
__device__ __forceinline__ long cache_row(const KvView& c, int page, int head, int slot) {
  return (((long)page * c.n_kv_heads + head) << c.page_shift) + slot;
}

// Lengths of sequence b as a kernel may use them: [q0, q0 + q_len) rows of the call, kv tokens in all, of which
// the first `held` have a place in the page table.  False (and reported): the sequence's entries make no sense.
constexpr long kMaxKvLen = 1L << 30;                          // key indexes stay well inside 32 bits
struct SeqLens { int q0, q_len, kv, held; };
__device__ __forceinline__ bool sequence_lengths(const BatchView& s, int b, int page_shift, int* status, SeqLens& o) {
  o.q0 = __ldg(s.q_start + b);
  const int q1 = __ldg(s.q_start + b + 1);
  o.kv = __ldg(s.kv_len + b);
  const long room = (long)s.max_pages << page_shift, capacity = room < kMaxKvLen ? room : kMaxKvLen;
  if (o.q0 < 0 || q1 < o.q0 || q1 > s.tokens || o.kv < 0) {
    report_device_error(status, HBL_ERR_RANGE);
    o.q_len = 0;
    o.held = 0;
    return false;
  }
  o.q_len = q1 - o.q0;
  o.held = o.kv;
  if (o.kv > capacity) {
    report_device_error(status, HBL_ERR_RANGE);
    o.held = (int)capacity;
  }
  return true;
}

// ---- launchers ---------------------------------------------------------------------------------------------------
int launch_rope_table(const double* freq, int n_freq, double amplitude, int first_pos, int n_pos, float* table, cudaStream_t s);
int launch_rope(const void* x, int dtype, int tokens, int n_heads, int head_dim, long x_ts, long x_hs, const int32_t* positions,
                const float* table, int n_pos, int rot_dim, int layout, int backward, void* out, long o_ts, long o_hs,
                cudaStream_t s);
int launch_kv_append(const KvView& c, const BatchView& b, const hbl_kv_append_t& a, cudaStream_t s);
int launch_kv_read(const KvView& c, const BatchView& b, void* k_out, void* v_out, cudaStream_t s);

struct AttnArgs {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  float* lse;
  long q_ts, q_hs, o_ts, o_hs;
  int n_heads, group, causal;
  float scale_log2;                    // sm_scale * log2(e): scores in units of log2
};
// How a call is split: the keys of a sequence go to `splits` thread blocks in pieces of `chunk`.
// The pieces' results wait in the workspace: `cap` rows (queries of one key head) for every sequence and key head from the
// streaming kernel, all rows of the call from the tiles.
struct AttnPlan { int splits, chunk, tiles, cap; };
struct AttnParts { float *rows_o, *rows_lse, *tiles_o, *tiles_lse; };      // [splits][rows][head_dim], [splits][rows]
// Sequences of up to `few` query rows (tokens times heads that share a key head) go to one kernel, the others to the other.
AttnPlan plan_attention_rows(const KvView& c, const BatchView& b, int n_heads, int few);
AttnPlan plan_attention_tiles(const KvView& c, const BatchView& b, int n_heads, int few);
int launch_attention_rows(const KvView& c, const BatchView& b, const AttnArgs& a, const AttnPlan& p, int few, const AttnParts& w,
                          bool beside_tiles, cudaStream_t s);
int launch_attention_tiles(const KvView& c, const BatchView& b, const AttnArgs& a, const AttnPlan& p, int few, const AttnParts& w,
                           cudaStream_t s);
int launch_attention_combine(const KvView& c, const BatchView& b, const AttnArgs& a, const AttnPlan& rows, const AttnPlan& tiles,
                             int few, const AttnParts& w, cudaStream_t s);

}  // namespace hbl
