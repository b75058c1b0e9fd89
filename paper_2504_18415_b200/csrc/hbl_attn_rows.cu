// Attention of few query rows over the paged cache: decoding steps.
//
//   s_j = sm_scale * ks_j * (q . ck_j),   p_j = 2^(s_j - m),   out = sum_j p_j vs_j cv_j / sum_j p_j
//
// bits 16: ck, cv are the bf16 values, the scales are 1 and p_j is rounded to bf16.  Codes are exact in fp16, and so are
// the queries once a row is scaled by a power of two; p_j vs_j is rounded to fp16 against a running power of two above
// the value scales.  These roundings are what the tensor core's operands cost; p's sum is taken before them, in fp32.
//
// The cache is read once per 8 (16) query rows of its key head.  bf16 is bound by that (one sequence of 131072 tokens: 91 us,
// 5.9 TB/s; 64 ragged ones of up to 4096 tokens 357).  Codes (64 x 4096 tokens of 32 key heads, one row: 4 bits 263 us, 4.3 TB/s;
// ragged 159) fill no unit: 60 % of the issue slots, 53 % of the logic pipe's cycles, 46 % of HBM's.  A thread block takes one
// (sequence, key head, row tile, piece of the keys), its four warps take 16 keys in turn and meet only at the end, so there
// is no barrier in the loop.  The keys are the M side of both products (S^T = K q^T, O^T = V^T P^T): 16 keys against 8
// rows, no half-empty tile, and a lane's operand registers are exactly the bytes that it loads from the cache
// (hbl_attn_frag.cuh), so nothing passes through shared memory but the queries.  The running maximum is only
// raised when a score exceeds it by more than 2^8 (p stays below 256): most steps rescale nothing and exchange nothing.
//
// Within a window (WINDOW) a block counts the keys that its rows see (KeyMap) and finds their pages from that; the rest is the same.
// 64 ragged sequences of up to 4096 tokens, window 1024, 4 bits: 87 us; what a block costs beside its keys is a third of that (27 us at
// a window of 64), so its chain is kept short: pages and the first token's rows are asked for before the queries, the
// warps' results lie side by side and are joined once (one warp after the other: 105 us).
#include "hbl_attn_frag.cuh"

namespace hbl {
namespace {

using namespace frag;

constexpr int kWarps = 4;
constexpr float kLazy = 8.f;

struct RowsParams {
  KvView c;
  BatchView b;
  AttnArgs a;
  AttnPlan p;
  float* part_o;                 // [splits][n_seqs * n_kv_heads * cap][head_dim], normalised; splits > 1 only
  float* part_lse;               // [splits][n_seqs * n_kv_heads * cap], log2 units
  int* status;
  int few;                       // sequences of more rows than this are another kernel's
  int ordered;                   // long sequences first
  int beside_tiles;              // launched behind the call's other kernel, of which it needs nothing
};

// The t-th sequence of the batch in falling order of their lengths' (or the window's) quarter of the longest.  The whole warp asks for the
// same t.  A batch of several rounds of blocks ends sooner when the long ones do not come last.
__device__ __forceinline__ int sequence_by_length(const BatchView& s, int reach, int t, int lane) {
  int most = 0;
  for (int b0 = 0; b0 < s.n_seqs; b0 += 32)
    if (b0 + lane < s.n_seqs) most = max(most, min(reach, __ldg(s.kv_len + b0 + lane)));
  most = __reduce_max_sync(0xffffffffu, most);
  const int step = most / 4 + 1;                               // lengths / step: 0 .. 3
  for (int quarter = 3; quarter >= 0; --quarter)
    for (int b0 = 0; b0 < s.n_seqs; b0 += 32) {
      const bool mine = b0 + lane < s.n_seqs && max(min(reach, __ldg(s.kv_len + min(b0 + lane, s.n_seqs - 1))), 0) / step == quarter;
      const unsigned hits = __ballot_sync(0xffffffffu, mine);
      const int n = __popc(hits);
      if (t < n) return b0 + __ffs(__ballot_sync(0xffffffffu, mine && __popc(hits & ((1u << lane) - 1)) == t)) - 1;
      t -= n;
    }
  return 0;                                                    // (not reached: every sequence is in one quarter)
}

template <int BITS, int D>
struct Geo {
  static constexpr int KU = D / 32, VU = D / 64;               // units of a key / value row a lane holds
  using KLane = Lane<BITS, KU, 4>;
  using VLane = Lane<BITS, VU, 8>;
  static constexpr int STEP_WORDS = 2 * KLane::WORDS + 4 * VLane::WORDS + 4;
  // steps whose loads are in flight ahead of the one at work, as far as registers go
  static constexpr int AHEAD = STEP_WORDS <= 40 ? 2 : 1;
  static constexpr int ROW_BYTES = D * BITS / 8;
};
template <int BITS, int D>
struct Step {
  typename Geo<BITS, D>::KLane k[2];
  typename Geo<BITS, D>::VLane v[4];
  float ks[2], vs[2];
};

// Thread blocks on an SM: what the registers of a block's accumulators and steps in flight leave.
constexpr int blocks_per_sm(int bits, int d, int nt) { return d > 128 ? 2 : nt == 1 ? 4 : bits < 16 ? 3 : 2; }

template <int BITS, int D, int NT, bool WINDOW, int W>
__global__ void __launch_bounds__(32 * W, blocks_per_sm(BITS, D, NT) * kWarps / W) attn_rows_kernel(const __grid_constant__ RowsParams p) {
  using G = Geo<BITS, D>;
  constexpr int ROWS = 8 * NT;
  constexpr int MT = D / 16;                                  // 16-element tiles of the output
  constexpr bool CODES = BITS < 16;
  __shared__ uint4 sq[NT][G::KU][32];
  __shared__ float sqs[ROWS];
  // Places for warps' results: one to a warp where there is room.  Two for 8-bit rows of 128, of which four blocks have 128 KB in flight:
  // shared memory comes out of the cache that their lanes' pieces of a row meet in (32 x 4096 tokens of 32 key heads: 239 us, with two or
  // one 229; 64 ragged 251, 245, 251; 8 x 2000 40.9, 39.8, 42.6; 4 x 509 11.7, 11.9, 13.4).
  constexpr int SLOTS = NT * D * W > 256 * 4 ? 1 : BITS == 8 && D == 128 && NT == 1 && W == 4 ? 2 : W;
  __shared__ __align__(16) float so[SLOTS][ROWS][D + 4];
  __shared__ float sm[W][ROWS], sl[W][ROWS], sv[W];
  // Behind the tiles this kernel begins when all their blocks have, so what came before the call is complete already; it
  // takes the SMs that they leave.  It may not be complete before they are, as what is launched next waits for this
  // kernel alone: its last block waits for them.
  const bool last = p.beside_tiles && blockIdx.x == gridDim.x - 1;
  if (!p.beside_tiles) grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  int id = blockIdx.x;
  const int split = id % p.p.splits; id /= p.p.splits;
  const int tile = id % p.p.tiles; id /= p.p.tiles;
  const int head = id % p.c.n_kv_heads;
  int b = id / p.c.n_kv_heads;
  if (p.ordered) b = sequence_by_length(p.b, p.p.reach, b, lane);
  SeqLens len;
  const bool sane = sequence_lengths(p.b, b, p.c.page_shift, p.status, len);
  const int group = p.a.group;
  const int n_rows = min(len.q_len, p.b.max_q_len) * group, r0 = tile * ROWS;
  if (!sane || r0 >= n_rows || n_rows > p.few || (split > 0 && (long)split * p.p.chunk >= min(len.held, p.p.reach))) {      // (no such piece: the combine step knows)
    if (last) grid_dependency_wait();
    return;
  }
  const int last_tok = min(r0 + ROWS - 1, n_rows - 1) / group;
  // keys any row of the tile sees (WINDOW: indexes of them, see KeyMap), and the piece of them that is this block's (the last
  // piece takes what is left)
  KeyMap map = {0, 0, 0};
  if (WINDOW) map = map_keys(p.a, len.kv - len.q_len + r0 / group);
  auto key_of = [&](int u) { return WINDOW && u >= map.sink_end ? u + map.gap : u; };
  const int past = len.kv - len.q_len - (WINDOW ? map.gap : 0);
  const int seen = p.a.causal ? max(0, min(len.held - (WINDOW ? map.gap : 0), past + last_tok + 1)) : len.held;
  const int key0 = split * p.p.chunk;
  int key1 = split == p.p.splits - 1 ? seen : min(seen, key0 + p.p.chunk);

  // ---- the keys, 16 at a time: the first loads, which take longest, before the queries.  All 16 rows of a step are read, those
  // beyond the last key too: a page is there as a whole, and what they hold is masked.  Row numbers fit 32 bits (checked on the
  // host): one multiply-add an address. ----
  const int* page_row = p.b.pages + (long)b * p.b.max_pages;
  Step<BITS, D> st[G::AHEAD];
  const unsigned char* kp = p.c.k + (g * G::ROW_BYTES);
  const unsigned char* vp = p.c.v + (2 * t * G::ROW_BYTES);
  const float* ksp = CODES ? p.c.k_scale + g : nullptr;
  const float* vsp = CODES ? p.c.v_scale + g : nullptr;
  const uint32_t page_rows = (uint32_t)p.c.n_kv_heads << p.c.page_shift, head_rows = (uint32_t)head << p.c.page_shift;
  const int slot_mask = (1 << p.c.page_shift) - 1;
  auto page_of = [&](int kb) { return kb < key1 ? __ldg(page_row + (key_of(kb) >> p.c.page_shift)) : -1; };
  auto load = [&](Step<BITS, D>& s, int kb, int page) {
    const bool here = page >= 0 && page < p.c.n_pages;         // (-1 beyond the last key)
    if (here) {
      const uint32_t row0 = (uint32_t)page * page_rows + head_rows + (uint32_t)(key_of(kb) & slot_mask);
      const unsigned char* k = kp + (uint64_t)row0 * G::ROW_BYTES;
      const unsigned char* v = vp + (uint64_t)row0 * G::ROW_BYTES;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s.k[h].load(k + 8 * h * G::ROW_BYTES, t);
        if (CODES) {
          s.ks[h] = __ldg(ksp + (uint64_t)row0 + 8 * h);
          s.vs[h] = __ldg(vsp + (uint64_t)row0 + 8 * h);
        }
      }
#pragma unroll
      for (int h = 0; h < 4; ++h) s.v[h].load(v + ((h & 1) + 8 * (h >> 1)) * G::ROW_BYTES, g);
    }
    return here;
  };
  constexpr int STRIDE = 16 * W;
  int kb = key0 + 16 * warp;
  int ahead_kb = kb, ahead_page = page_of(kb);
  // The first token at 8 bits: by the warp whose turn key 0 is, or, within a window, by the one that has least to do; its rows
  // are asked for here.
  const bool bos = BITS < 8 && p.c.bos_k != nullptr && (!WINDOW || p.a.sinks > 0 || (map.first | map.gap) == 0);
  constexpr int BOS_WARP = WINDOW ? W - 1 : 0;
  int bos_row = -1;
  if (bos && key0 == 0 && key1 > 0) {
    const int slot = p.b.bos_slot != nullptr ? __ldg(p.b.bos_slot + b) : b;
    if (slot >= 0 && slot < p.c.n_slots) bos_row = slot;
    else report_device_error(p.status, HBL_ERR_RANGE);        // its first token is then left out
  }
  uint2 bos_k[BITS < 8 ? G::KU : 1], bos_v[BITS < 8 ? G::VU : 1];
  float bos_ks = 0.f, bos_vs = 0.f;
  if constexpr (BITS < 8) {
    if (bos_row >= 0 && warp == BOS_WARP) {
      const long brow = (long)bos_row * p.c.n_kv_heads + head;
#pragma unroll
      for (int i = 0; i < G::KU; ++i) bos_k[i] = __ldg(reinterpret_cast<const uint2*>(p.c.bos_k + brow * D) + G::KLane::unit_of(i, t));
#pragma unroll
      for (int i = 0; i < G::VU; ++i) bos_v[i] = __ldg(reinterpret_cast<const uint2*>(p.c.bos_v + brow * D) + G::VLane::unit_of(i, g));
      bos_ks = __ldg(p.c.bos_k_scale + brow);
      bos_vs = __ldg(p.c.bos_v_scale + brow);
    }
  }

  // ---- queries as B fragments: row n = g of tile nt, its pairs in the order the keys' units have.  For codes they are
  // fp16, scaled by the power of two that brings the row's largest magnitude near 2^15: a bf16 value keeps all its bits
  // down to 2^-29 of that.  A warp takes whole rows. ----
#pragma unroll
  for (int i = 0; i < ROWS / W; ++i) {
    const int rr = warp + i * W, r = r0 + rr, nt = rr >> 3;
    constexpr int CH = D / 8, PER = CH > 32 ? CH / 32 : 1;     // 16-byte pieces of a row: one to a lane
    static_assert(PER == 1, "a row is at most 32 pieces");
    uint4 w = make_uint4(0, 0, 0, 0);
    if (r < n_rows && lane < CH) {
      const int tok = r / group, hq = head * group + r % group;
      w = __ldg(reinterpret_cast<const uint4*>(p.a.q + (len.q0 + tok) * p.a.q_ts + hq * p.a.q_hs + 8 * lane));
    }
    uint32_t x[4] = {w.x, w.y, w.z, w.w};
    if (CODES) {
      uint32_t top = 0;                                        // exponent of the largest finite magnitude
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = x[j] << 16 & 0x7F800000u, hi = x[j] & 0x7F800000u;
        top = max(top, max(lo == 0x7F800000u ? 0u : lo, hi == 0x7F800000u ? 0u : hi));
      }
      top = __reduce_max_sync(0xffffffffu, top) >> 23;
      // times 2^(14 - (top - 127)), in two steps that stay in range; back by the inverse
      const int up = top == 0 ? 0 : 141 - (int)top;
      const float f0 = __uint_as_float((uint32_t)(127 + up / 2) << 23), f1 = __uint_as_float((uint32_t)(127 + up - up / 2) << 23);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        x[j] = pack2_f16(__uint_as_float(x[j] << 16) * f0 * f1, __uint_as_float(x[j] & 0xFFFF0000u) * f0 * f1);
      if (lane == 0) sqs[rr] = p.a.scale_log2 * (1.f / f0) * (1.f / f1);
    } else if (lane == 0) {
      sqs[rr] = p.a.scale_log2;
    }
    if (lane < CH) {
      uint32_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int lo = pair16_lo<BITS>(j), hi = pair16_hi<BITS>(j);
        o[j] = __byte_perm(x[lo / 2], x[hi / 2], (lo & 1 ? 0x32 : 0x10) | (hi & 1 ? 0x7600 : 0x5400));
      }
      // which lane of the row's four, and which of its units, this piece is
#pragma unroll
      for (int u = 0; u < G::KU; ++u)
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
          if (G::KLane::unit_of(u, tt) == lane) sq[nt][u][(rr & 7) * 4 + tt] = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
  __syncthreads();

  // rows of this lane's score columns: 2t and 2t + 1 of every tile; they see keys below lim
  int lim[NT][2], low = 0x7fffffff;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = r0 + nt * 8 + 2 * t + e;
      lim[nt][e] = r >= n_rows ? 0 : p.a.causal ? past + r / group + 1 : seen;
      if (r < n_rows) low = min(low, lim[nt][e]);
    }
  low = min(low, key1);
  low = __reduce_min_sync(0xffffffffu, low);                  // below it no key needs a mask ...
  const int expired = past + last_tok + 1 - p.a.window;       // ... WINDOW: but for those below this that are no sinks

  // Per column: minus the maximum so far (0: none yet), p's sum.  `some`: every column has a maximum.
  // vr: a power of two no smaller than any value scale so far.  The weights go to the tensor core as p vs / vr * 2^7 in
  // fp16: at most 2^15, rounded by 2^-11 of themselves, or by 2^-32 vr where they are that small.
  float neg[NT][2], qs[NT][2], l[NT][2], o[NT][MT][4];
  float vr = 0x1p-100f, inv_vr = 0x1p107f;
  uint32_t poison = 0;                                         // bits 16: columns that saw a masked step's value that is not finite
  uint32_t some = 0;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      neg[nt][e] = 0.f;
      l[nt][e] = 0.f;
      qs[nt][e] = sqs[nt * 8 + 2 * t + e];
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.f;
  }

  // scores (c: keys g and g + 8, columns 2t and 2t + 1) to P^T fragments, with the running maximum.
  // masked: keys beyond a column's limit, or before its window, and key 0 where skip_first, do not count.
  auto softmax = [&](float (&c)[NT][4], int kb, const float (&ks)[2], const float (&vs)[2], bool masked, bool skip_first,
                     uint32_t (&pf)[NT][2]) {
    float top = -INFINITY;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (CODES) c[nt][e] *= qs[nt][e & 1];
        c[nt][e] = fmaf(c[nt][e], CODES ? ks[e >> 1] : qs[nt][e & 1], neg[nt][e & 1]);
        if (masked) {
          const int key = kb + g + (e >> 1) * 8;
          if (key >= min(lim[nt][e & 1], key1) || (skip_first && key == 0)) c[nt][e] = -INFINITY;
          if (WINDOW && key >= p.a.sinks && key < lim[nt][e & 1] - p.a.window) c[nt][e] = -INFINITY;
        }
        top = fmaxf(top, c[nt][e]);
      }
    const bool wide = CODES && fmaxf(fabsf(vs[0]), fabsf(vs[1])) > vr;       // (a scale that is not finite never counts, see vf)
    if (__any_sync(0xffffffffu, top > (some ? kLazy : -INFINITY) || wide)) {
      float fv = 1.f;
      if (CODES) {
        uint32_t v = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t x = __float_as_uint(fabsf(vs[h]));
          const int key = kb + g + 8 * h;
          if (x < 0x7F000000u && key < key1 && (!WINDOW || key >= map.first || key < p.a.sinks)) v = max(v, x);
        }
        v = (__reduce_max_sync(0xffffffffu, v) + 0x7FFFFFu) & 0x7F800000u;
        const float to = fmaxf(vr, __uint_as_float(v));
        fv = vr / to;                                          // a power of two (0 where it leaves the range)
        vr = to;
        inv_vr = 128.f / to;
      }
      bool all = true;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = fmaxf(c[nt][e], c[nt][e + 2]);
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
          const bool old = l[nt][e] != 0.f || neg[nt][e] != 0.f;     // (this lane's part of a sum may be 0 after a first key)
          const bool seen = (__ballot_sync(0xffffffffu, old) & (0x11111111u << t)) != 0;
          const float by = x > (seen ? kLazy : -INFINITY) ? x : 0.f;
          f[e] = seen ? exp2_approx(-by) : 0.f;
          neg[nt][e] -= by;
          c[nt][e] -= by;
          c[nt][e + 2] -= by;
          l[nt][e] *= f[e];
          all = all && (seen || x > -INFINITY);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          o[nt][i][0] *= f[0] * fv; o[nt][i][1] *= f[1] * fv; o[nt][i][2] *= f[0] * fv; o[nt][i][3] *= f[1] * fv;
        }
      }
      some = __all_sync(0xffffffffu, all);
    }
    // (0 * a scale that is not finite is NaN: its weight is, so every element of a row that sees its key is, too)
    const float vf[2] = {fmaf(vs[0], 0.f, vs[0] * inv_vr), fmaf(vs[1], 0.f, vs[1] * inv_vr)};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = exp2_approx(c[nt][e]);
        l[nt][e & 1] += x;
        w[e] = CODES ? x * vf[e >> 1] : x;
        if (masked && c[nt][e] == -INFINITY) w[e] = 0.f;        // (a scale that is not finite stays out, too)
      }
      pf[nt][0] = transpose8x8(CODES ? pack2_f16(w[0], w[1]) : pack2(w[0], w[1]));
      pf[nt][1] = transpose8x8(CODES ? pack2_f16(w[2], w[3]) : pack2(w[2], w[3]));
    }
  };

  // ---- the first token at 8 bits: one key ----
  if constexpr (BITS < 8) {
    if (bos_row >= 0 && warp == BOS_WARP) {
      auto value = [](const uint2& u, int e) { return (float)((int)(((e < 4 ? u.x : u.y) >> (8 * (e & 3))) & 255u) - 128); };
      float c[NT][4] = {};
#pragma unroll
      for (int i = 0; i < G::KU; ++i) {
        uint32_t a[4] = {0, 0, 0, 0};
        if (g == 0) {
          const uint2 u = bos_k[i];
#pragma unroll
          for (int j = 0; j < 4; ++j) a[j] = pack2_f16(value(u, pair16_lo<BITS>(j)), value(u, pair16_hi<BITS>(j)));
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint4 q = sq[nt][i][lane];
          mma_rows<BITS>(c[nt], a[0], 0, a[1], 0, q.x, q.y);
          mma_rows<BITS>(c[nt], a[2], 0, a[3], 0, q.z, q.w);
        }
      }
      // key 0 alone: the other rows of the step are put out of it
      const float ks[2] = {bos_ks, 0.f}, vs[2] = {g == 0 ? bos_vs : 0.f, 0.f};
      const int whole = key1;
      key1 = 1;
      uint32_t pf[NT][2];
      softmax(c, 0, ks, vs, true, false, pf);
      key1 = whole;
#pragma unroll
      for (int i = 0; i < G::VU; ++i) {
        uint32_t a[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (t == 0) {
          const uint2 u = bos_v[i];
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] = pack2_f16(value(u, e), 0.f);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int q = 0; q < 4; ++q) mma_rows<BITS>(o[nt][4 * i + q], a[2 * q], a[2 * q + 1], 0, 0, pf[nt][0], pf[nt][1]);
      }
    }
  }

  // ---- the keys ----
  bool here[G::AHEAD];
#pragma unroll
  for (int d = 0; d < G::AHEAD; ++d) {
    here[d] = load(st[d], ahead_kb, ahead_page);
    ahead_kb += STRIDE;
    ahead_page = page_of(ahead_kb);
  }
  while (kb < key1) {
#pragma unroll
    for (int d = 0; d < G::AHEAD; ++d) {
      if (kb < key1) {
        Step<BITS, D>& s = st[d];
        if (!here[d]) {
          report_device_error(p.status, HBL_ERR_RANGE);
        } else {
          const bool masked = kb + 16 > low || (bos && kb == 0) || (WINDOW && kb < expired && kb + 16 > p.a.sinks);
          if (!CODES && masked) {
            // 0 * a value that is not finite would reach the columns it is masked for: such values become zeros, and the
            // columns that do see their key are marked; what lies beyond the last key becomes zeros, whatever it is
            uint32_t bad = 0;                                  // keys of the step
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              const int r = 2 * t + (h & 1) + 8 * (h >> 1);
              bool any = false;
#pragma unroll
              for (int i = 0; i < G::VLane::WORDS; ++i) {
                const uint32_t x = s.v[h].w[i];
                any |= (x & 0x7F800000u) == 0x7F800000u || (x & 0x7F80u) == 0x7F80u;
              }
              if (any || kb + r >= key1) s.v[h].clear();
              if (any && kb + r < key1) bad |= 1u << r;
            }
            bad = __reduce_or_sync(0xffffffffu, bad);
            if (bad != 0) {
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  auto below = [&](int u) { return u >= kb + 16 ? 0xFFFFu : u > kb ? (1u << (u - kb)) - 1 : 0u; };
                  uint32_t visible = below(min(lim[nt][e], key1));
                  if (WINDOW) visible &= ~below(lim[nt][e] - p.a.window) | below(p.a.sinks);
                  if (bad & visible) poison |= 1u << (2 * nt + e);
                }
            }
          }
          float c[NT][4] = {};
#pragma unroll
          for (int i = 0; i < G::KU; ++i) {
            uint32_t x[4], y[4];
            pairs16<BITS>(s.k[0], i, t, x);
            pairs16<BITS>(s.k[1], i, t, y);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const uint4 q = sq[nt][i][lane];
              mma_rows<BITS>(c[nt], x[0], y[0], x[1], y[1], q.x, q.y);
              mma_rows<BITS>(c[nt], x[2], y[2], x[3], y[3], q.z, q.w);
            }
          }
          uint32_t pf[NT][2];
          softmax(c, kb, s.ks, s.vs, masked, bos, pf);
#pragma unroll
          for (int i = 0; i < G::VU; ++i) {
            uint32_t x[8], y[8];
            cross16<BITS>(s.v[0], s.v[1], i, g, x);
            cross16<BITS>(s.v[2], s.v[3], i, g, y);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int q = 0; q < 4; ++q)
                mma_rows<BITS>(o[nt][4 * i + q], x[2 * q], x[2 * q + 1], y[2 * q], y[2 * q + 1], pf[nt][0], pf[nt][1]);
          }
        }
      }
      here[d] = load(st[d], ahead_kb, ahead_page);
      ahead_kb += STRIDE;
      ahead_page = page_of(ahead_kb);
      kb += STRIDE;
    }
  }

  // ---- the warps' results together ----
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float x = l[nt][e];
      x += __shfl_xor_sync(0xffffffffu, x, 4);
      x += __shfl_xor_sync(0xffffffffu, x, 8);
      x += __shfl_xor_sync(0xffffffffu, x, 16);
      if (!CODES && (poison >> (2 * nt + e) & 1)) {
#pragma unroll
        for (int i = 0; i < MT; ++i) o[nt][i][e] = o[nt][i][e + 2] = __uint_as_float(0x7FC00000u);
      }
      if (g == 0) {
        sm[warp][nt * 8 + 2 * t + e] = x == 0.f ? -INFINITY : -neg[nt][e];     // (a NaN has a place in the sum, too)
        sl[warp][nt * 8 + 2 * t + e] = x;
      }
    }
  if (lane == 0) sv[warp] = CODES ? vr * 0x1p-7f : 1.f;
  // a warp's maximum, and what its results are in units of, against those of all: (0 where there was no key)
  auto top_of = [&](int r) {
    float top = sm[0][r];
#pragma unroll
    for (int w = 1; w < W; ++w) top = fmaxf(top, sm[w][r]);
    return top;
  };
  auto share = [&](int w, int r, float top) { return exp2_approx(sm[w][r] - (top == -INFINITY ? 0.f : top)); };
  auto put = [&](float (&to)[ROWS][D + 4], bool first, const float (&f)[NT][2]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int d = 8 * G::VLane::unit_of(i / 4, g) + 2 * (i & 3) + (e >> 1);
          float& x = to[nt * 8 + 2 * t + (e & 1)][d];
          const float y = o[nt][i][e] * f[nt][e & 1];
          x = first ? y : x + y;
        }
  };
  if constexpr (SLOTS == W) {                                  // side by side, joined by who writes them out
    float one[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) one[nt][0] = one[nt][1] = 1.f;
    put(so[warp], true, one);
    __syncthreads();
  } else {                                                     // as many as there are places, and the next on top of them
    __syncthreads();
    float f[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = nt * 8 + 2 * t + e;
        f[nt][e] = share(warp, r, top_of(r)) * sv[warp];
      }
    for (int w = 0; w < W; w += SLOTS) {
      if (warp / SLOTS * SLOTS == w) put(so[warp % SLOTS], w == 0, f);
      __syncthreads();
    }
  }
  const long all_rows = (long)p.b.n_seqs * p.c.n_kv_heads * p.p.cap;
  for (int i = threadIdx.x; i < ROWS * (D / 4); i += 32 * W) {
    const int rr = i / (D / 4), d = (i % (D / 4)) * 4, r = r0 + rr;
    if (r >= n_rows) break;
    const float top = top_of(rr);
    float4 v = *reinterpret_cast<const float4*>(&so[0][rr][d]);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = share(w, rr, top);
      sum += sl[w][rr] * f;
      if constexpr (SLOTS == W) {
        const float4 x = *reinterpret_cast<const float4*>(&so[w][rr][d]);
        const float by = f * sv[w];
        if (w == 0) {
          v = make_float4(x.x * by, x.y * by, x.z * by, x.w * by);
        } else {
          v.x += x.x * by; v.y += x.y * by; v.z += x.z * by; v.w += x.w * by;
        }
      }
    }
    if constexpr (SLOTS < W)
#pragma unroll
      for (int w = 1; w < SLOTS; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(&so[w][rr][d]);
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
      }
    const float inv = sum == 0.f ? 0.f : __fdividef(1.f, sum);
    const int tok = len.q0 + r / group, hq = head * group + r % group;
    const float lse2 = sum == 0.f ? -INFINITY : top + __log2f(sum);
    if (p.p.splits > 1) {
      const long row = split * all_rows + ((long)b * p.c.n_kv_heads + head) * p.p.cap + r;
      *reinterpret_cast<float4*>(p.part_o + row * D + d) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
      if (d == 0) p.part_lse[row] = lse2;
    } else {
      *reinterpret_cast<uint2*>(p.a.out + tok * p.a.o_ts + hq * p.a.o_hs + d) =
          make_uint2(pack2(v.x * inv, v.y * inv), pack2(v.z * inv, v.w * inv));
      if (d == 0 && p.a.lse != nullptr) p.a.lse[(long)tok * p.a.n_heads + hq] = lse2 * 0.6931471805599453f;
    }
  }
  if (last) grid_dependency_wait();
}

// The pieces of a row together (whichever kernel computed them): out = sum_s 2^(lse_s - top) o_s / sum_s 2^(lse_s - top).
// The streaming kernel's rows are dealt to the warps by sequence, key head and row; where the tiles are split, too, all rows
// of the call are.  (Looking every row up cost 161 us on four 2048-token prompts, none of which was split.)
// `share` warps (1, 2, 4 or 8, by the number of pieces) take the pieces of a row in turn, four loads in flight each, and
// add up through shared memory in a fixed order.
struct CombineParams {
  KvView c;
  BatchView b;
  AttnArgs a;
  AttnPlan rows, tiles;          // of sequences of up to `few` rows, and of the others
  int few, share, short_only;
  AttnParts w;
  int* status;
};
template <int D>
__global__ void __launch_bounds__(256) attn_combine_kernel(const __grid_constant__ CombineParams p) {
  constexpr int E = D / 32;
  __shared__ float s_acc[8][D], s_sum[8];
  grid_dependency_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = warp % p.share;
  const long unit = ((long)blockIdx.x * 8 + warp) / p.share, short_rows = (long)p.b.n_seqs * p.c.n_kv_heads * p.rows.cap;
  const long call_rows = (long)p.b.tokens * p.a.n_heads;
  int tok = 0, hq = 0, pieces = 0;                            // pieces 0: nothing to do
  const float *part_o = nullptr, *part_lse = nullptr;
  long row = 0, total_rows = 0;                               // in the parts
  auto pieces_of = [&](const AttnPlan& plan, const SeqLens& len) {
    const int held = min(len.held, plan.reach);
    return plan.splits > 1 ? max(1, min(plan.splits, (held + plan.chunk - 1) / plan.chunk)) : 0;      // (0: written whole)
  };
  SeqLens len;
  int b = p.b.n_seqs;
  if (p.short_only && unit < short_rows) {
    b = (int)(unit / (p.c.n_kv_heads * p.rows.cap));
    const int r = (int)(unit % p.rows.cap);
    if (sequence_lengths(p.b, b, p.c.page_shift, p.status, len) && r < min(len.q_len, p.b.max_q_len) * p.a.group) {
      tok = len.q0 + r / p.a.group;
      hq = (int)(unit / p.rows.cap % p.c.n_kv_heads) * p.a.group + r % p.a.group;
    } else {
      b = p.b.n_seqs;
    }
  } else if (!p.short_only && unit < call_rows) {
    tok = (int)(unit / p.a.n_heads);
    hq = (int)(unit % p.a.n_heads);
    b = find_sequence(p.b.q_start, p.b.n_seqs, tok, lane);
    if (b < p.b.n_seqs && !(sequence_lengths(p.b, b, p.c.page_shift, p.status, len) && tok >= len.q0 && tok - len.q0 < p.b.max_q_len)) b = p.b.n_seqs;
  }
  if (b < p.b.n_seqs) {
    if ((long)min(len.q_len, p.b.max_q_len) * p.a.group > p.few) {
      pieces = pieces_of(p.tiles, len);
      part_o = p.w.tiles_o;
      part_lse = p.w.tiles_lse;
      row = (long)tok * p.a.n_heads + hq;
      total_rows = call_rows;
    } else {
      pieces = pieces_of(p.rows, len);
      part_o = p.w.rows_o;
      part_lse = p.w.rows_lse;
      row = ((long)b * p.c.n_kv_heads + hq / p.a.group) * p.rows.cap + (tok - len.q0) * p.a.group + hq % p.a.group;
      total_rows = short_rows;
    }
  }
  float top = -INFINITY;
  for (int s = lane; s < pieces; s += 32) top = fmaxf(top, part_lse[s * total_rows + row]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  float acc[E] = {}, sum = 0.f;
  for (int s0 = mine; s0 < pieces; s0 += 4 * p.share) {
    float w[4], v[4][E];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int s = s0 + k * p.share;
      const float x = s < pieces ? part_lse[s * total_rows + row] : -INFINITY;
      w[k] = x == -INFINITY ? 0.f : exp2_approx(x - top);     // (a NaN stays one)
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = 0.f;
      if (s < pieces) {
        const float* src = part_o + (s * total_rows + row) * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 y = *reinterpret_cast<const float2*>(src + e);
          v[k][e] = y.x;
          v[k][e + 1] = y.y;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      sum += w[k];
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += w[k] * v[k][e];    // (a piece without a key holds zeros)
    }
  }
  if (p.share > 1) {
    if (lane == 0) s_sum[warp] = sum;
#pragma unroll
    for (int e = 0; e < E; ++e) s_acc[warp][lane * E + e] = acc[e];
    __syncthreads();
    if (mine != 0) return;
    for (int w = 1; w < p.share; ++w) {
      sum += s_sum[warp + w];
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += s_acc[warp + w][lane * E + e];
    }
  }
  if (pieces == 0) return;
  const float inv = sum == 0.f ? 0.f : __fdividef(1.f, sum);
  uint32_t* dst = reinterpret_cast<uint32_t*>(p.a.out + tok * p.a.o_ts + hq * p.a.o_hs + lane * E);
#pragma unroll
  for (int e = 0; e < E; e += 2) dst[e / 2] = pack2(acc[e] * inv, acc[e + 1] * inv);
  if (lane == 0 && p.a.lse != nullptr) p.a.lse[(long)tok * p.a.n_heads + hq] = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * 0.6931471805599453f;
}

long most_rows(const BatchView& b, int group, int few) {
  const long rows = (long)b.max_q_len * group;                // (few is the border, not the most: above it the other kernel works)
  return rows < few ? rows : few;
}
int rows_per_tile(const BatchView& b, int group, int few) { return most_rows(b, group, few) > 8 ? 16 : 8; }

template <int BITS, int D, bool WINDOW>
int launch_rows_dim(RowsParams& p, cudaStream_t s) {
  const long blocks = (long)p.b.n_seqs * p.c.n_kv_heads * p.p.tiles * p.p.splits;
  if (blocks > 0x7fffffffL) return HBL_ERR_TOO_LARGE;
  const bool narrow = rows_per_tile(p.b, p.a.group, p.few) == 8;
  // Within a window: eight warps where every block has an SM to itself (4 x 509 tokens at 8 bits, window of 128: 7.1 us, with four
  // 8.5; of 500: 9.5, 12.6; 64 x 4096 tokens, of 1024: 107, 94), as far as there is room for their results.
  if constexpr (WINDOW && D <= 128) {
    if (blocks <= sm_count() && (narrow || D <= 64)) {
      if (narrow) HBL_CUDA_OK(launch_waiting(attn_rows_kernel<BITS, D, 1, WINDOW, 8>, dim3((unsigned)blocks), dim3(256), 0, s, p));
      else HBL_CUDA_OK(launch_waiting(attn_rows_kernel<BITS, D, D <= 64 ? 2 : 1, WINDOW, 8>, dim3((unsigned)blocks), dim3(256), 0, s, p));
      note_launch();
      return HBL_OK;
    }
  }
  if (narrow)
    HBL_CUDA_OK(launch_waiting(attn_rows_kernel<BITS, D, 1, WINDOW, kWarps>, dim3((unsigned)blocks), dim3(32 * kWarps), 0, s, p));
  else
    HBL_CUDA_OK(launch_waiting(attn_rows_kernel<BITS, D, 2, WINDOW, kWarps>, dim3((unsigned)blocks), dim3(32 * kWarps), 0, s, p));
  note_launch();
  return HBL_OK;
}
template <int BITS, bool WINDOW>
int launch_rows_window(RowsParams& p, cudaStream_t s) {
  switch (p.c.head_dim) {
    case 64: return launch_rows_dim<BITS, 64, WINDOW>(p, s);
    case 128: return launch_rows_dim<BITS, 128, WINDOW>(p, s);
    case 256: return launch_rows_dim<BITS, 256, WINDOW>(p, s);
    default: return HBL_ERR_SHAPE;
  }
}
template <int BITS>
int launch_rows_bits(RowsParams& p, cudaStream_t s) {
  return p.a.window > 0 ? launch_rows_window<BITS, true>(p, s) : launch_rows_window<BITS, false>(p, s);
}

// How many pieces the keys of a sequence are dealt in.
//   None up to 512 keys, where the second launch costs more than the shorter loops save (4 x 509 tokens: 11.2 us in two
// pieces, 9.6 in one; 4 x 1000: 14.1, 14.0), and none of less than 256 keys.
//   Few sequences: as many pieces as there is room for at once; with one more the last waits for a whole round (16 rows
// over 16384 tokens at 8 bits: 57 us in 13 pieces, 70 in 14).
//   As many as there is room for, or more: whole (32 x 4096 tokens of 32 key heads at 8 bits, ragged with one row: 106 us, in two
// pieces 115; not always: 16 rows each 382, 361).
//   In between the host, which does not know the lengths, weighs two batches: every sequence as long as the bound says
// (whole rounds of resident blocks; a round that is not full costs half of one and its part of the other half), and
// lengths anywhere below it (the work, evenly spread, and half of a last piece), which is what it mostly is, so that it
// counts twice.  A block costs as much as `fixed` keys before its first and after its last one (64 x 4096 tokens at 4 bits
// in 1, 2, 4, 8 pieces: 264, 274, 302, 358 us).  64 ragged sequences of up to 16384 tokens, 8 key heads, 4 bits: 252 us in 1
// piece, 189 in 2, 162 in 4, 159 in 8, 174 in 16.
long pieces_of_keys(long base, int resident, long keys, long most, int bits) {
  const long slots = (long)sm_count() * resident;
  if (base <= 0 || most <= 1 || base >= slots) return 1;
  if (8 * base <= slots) return slots / base < most ? slots / base : most;
  const float fixed = bits == 16 ? 300.f : 600.f, load = (float)base / (float)slots;
  long best = 1;
  float least = 0.f;
  for (long n = 1; n <= most && n <= 16; ++n) {
    const long on_sm = (n * base + sm_count() - 1) / sm_count(), rest = on_sm % resident;
    const float piece = (float)keys / (float)n + fixed;
    const float even = ((float)(on_sm / resident) + (rest > 0 ? 0.5f + 0.5f * (float)rest / (float)resident : 0.f)) * piece;
    const float uneven = load * 0.5f * ((float)keys + fixed * (float)(n + 1)) + 0.5f * piece;
    if (n == 1 || even + 2.f * uneven < least) {
      best = n;
      least = even + 2.f * uneven;
    }
  }
  return best;
}

}  // namespace

int attention_rows_resident(const KvView& c, const BatchView& b, const AttnArgs& a, int few) {
  return blocks_per_sm(c.bits, c.head_dim, rows_per_tile(b, a.group, few) / 8);
}

AttnPlan plan_attention_rows(const KvView& c, const BatchView& b, const AttnArgs& a, int few) {
  AttnPlan p{};
  const int group = a.group, rows = rows_per_tile(b, group, few);
  p.cap = (int)most_rows(b, group, few);
  p.tiles = (p.cap + rows - 1) / rows;
  p.reach = reach_of(a, rows);
  const long base = (long)b.n_seqs * c.n_kv_heads * p.tiles, keys = b.max_kv_len < p.reach ? b.max_kv_len : p.reach;
  const long most = keys <= 512 ? 1 : (keys + 255) / 256;
  const long n = pieces_of_keys(base, blocks_per_sm(c.bits, c.head_dim, rows / 8), keys, most, c.bits);
  p.chunk = (int)(((keys + n - 1) / n + 63) / 64 * 64);
  if (p.chunk < 64) p.chunk = 64;
  p.splits = (int)((keys + p.chunk - 1) / p.chunk);
  if (p.splits < 1) p.splits = 1;
  return p;
}

int launch_attention_rows(const KvView& c, const BatchView& b, const AttnArgs& a, const AttnPlan& plan, int few, const AttnParts& w,
                          bool beside_tiles, cudaStream_t s) {
  RowsParams p{};
  p.c = c; p.b = b; p.a = a; p.p = plan; p.few = few; p.part_o = w.rows_o; p.part_lse = w.rows_lse;
  p.beside_tiles = beside_tiles;
  // More blocks than fit at once, of whole sequences: the long ones first (64 ragged sequences of up to 4096 tokens at 4 bits
  // 178 us in the batch's order, 159 in this; 128 of 8 key heads 99, 82; all of one length 260, 263; window of 1024, ragged 88, 87, of
  // 2048 138, 131).  Not for short ones, whose blocks would spend more on the look-up than it saves (up to 600 tokens: 41 us, 44;
  // window of 256: 41, 44), nor for batches whose look-up is long.
  const long slots = (long)sm_count() * attention_rows_resident(c, b, a, few);
  p.ordered = plan.splits == 1 && (b.max_kv_len < plan.reach ? b.max_kv_len : plan.reach) >= 1024 && b.n_seqs <= 128 && (long)b.n_seqs * c.n_kv_heads * plan.tiles > slots;
  p.status = device_status_word();
  if (p.status == nullptr) return HBL_ERR_CUDA;
  switch (c.bits) {
    case 3: return launch_rows_bits<3>(p, s);
    case 4: return launch_rows_bits<4>(p, s);
    case 8: return launch_rows_bits<8>(p, s);
    case 16: return launch_rows_bits<16>(p, s);
    default: return HBL_ERR_BITS;
  }
}

int launch_attention_combine(const KvView& c, const BatchView& b, const AttnArgs& a, const AttnPlan& rows, const AttnPlan& tiles,
                             int few, const AttnParts& w, cudaStream_t s) {
  CombineParams p{};
  p.c = c; p.b = b; p.a = a; p.rows = rows; p.tiles = tiles; p.few = few; p.w = w;
  p.status = device_status_word();
  if (p.status == nullptr) return HBL_ERR_CUDA;
  const int most = rows.splits > tiles.splits ? rows.splits : tiles.splits;
  p.share = most <= 4 ? 1 : most <= 8 ? 2 : most <= 16 ? 4 : 8;
  p.short_only = tiles.splits <= 1;
  const long units = p.short_only ? (long)b.n_seqs * c.n_kv_heads * rows.cap : (long)b.tokens * a.n_heads;
  const long blocks = (units * p.share + 7) / 8;
  if (blocks > 0x7fffffffL) return HBL_ERR_TOO_LARGE;
  const dim3 grid((unsigned)blocks), block(256);
  switch (c.head_dim) {
    case 64: HBL_CUDA_OK(launch_waiting(attn_combine_kernel<64>, grid, block, 0, s, p)); break;
    case 128: HBL_CUDA_OK(launch_waiting(attn_combine_kernel<128>, grid, block, 0, s, p)); break;
    case 256: HBL_CUDA_OK(launch_waiting(attn_combine_kernel<256>, grid, block, 0, s, p)); break;
    default: return HBL_ERR_SHAPE;
  }
  note_launch();
  return HBL_OK;
}

}  // namespace hbl
