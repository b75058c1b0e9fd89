// The paged cache of attention states: tokens into it (keys rotated, keys and values quantized per head, queries
// rotated, all in one launch) and out of it as bf16 values.
//
//   gamma = max_d |x[d]|,  u = round((2^(b-1) - 1) / (gamma + eps) * x) + 2^(b-1),  scale = gamma / (2^(b-1) - 1)
//
// Prompts: 2 bytes read and b / 8 written per element, queries 2 and 2.  bf16 rows are bound by HBM (four 2048-token
// prompts of 96 heads with reading them back: 72 us, 5.6 TB/s), codes by the issue of instructions (78 % of the slots at 3
// bits: widening, rotation, the maximum's shuffles, packing, and choosing what each head is; 147 us, 2.9 TB/s).  Append and read
// apart, 3, 4, 8, 16 bits: 113, 103, 104, 78 us and 47, 45, 41, 49.  A decoding step (64 tokens of 96 heads: 4.0 us and 2.2 us in
// a replayed graph) is bound by the chain of dependent loads (sequence -> length -> page -> row).  A lane owns 8 consecutive elements of a head, so a head
// is head_dim / 8 lanes and its maximum takes three to five shuffles; the partner of a rotated element lies in the same
// lane (interleaved layout) or one shuffle away (half layout).  A thread takes ROWS heads of the same token: the table's
// pairs are loaded once for all of them, and their loads are in flight together.  The loads of the data depend on the
// number of rows that there are, but not on that chain, and are issued before it.
// With norms (hbl_kv_append_norm): four prompts of 32 and 2 x 32 heads, read back, 3, 4, 8, 16 bits: 181, 175, 167, 98 us; 76 % of the issue
// slots.  Squares and one root to a head: each lane adds up one of its ROWS heads and takes its root (every lane all of them: 212 us).
#include "hbl_kv_cache.cuh"
#include "hbl_piece.cuh"

namespace hbl {
namespace {

constexpr int kThreads = 256;
constexpr float kMagic = 12582912.0f;                        // 1.5 * 2^23: x + kMagic has rint(x) in its low mantissa bits

__device__ __forceinline__ void widen8(const uint4& raw, float (&f)[8]) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 narrow8(const float (&f)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ uint32_t low_bytes(uint32_t u0, uint32_t u1, uint32_t u2, uint32_t u3) {
  return __byte_perm(__byte_perm(u0, u1, 0x0040), __byte_perm(u2, u3, 0x0040), 0x5410);
}
// Unsigned codes of 8 elements as bytes.  |f| <= gamma, so |rq f| < c and no clip is needed; a head that is not
// finite comes with rq = 0 and f = 0, i.e. with the code of zero.
template <int BITS>
__device__ __forceinline__ uint2 codes8(const float (&f)[8], float rq) {
  uint32_t u[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(__fadd_rn(__fmul_rn(rq, f[i]), kMagic + (float)(1 << (BITS - 1))));
  return make_uint2(low_bytes(u[0], u[1], u[2], u[3]), low_bytes(u[4], u[5], u[6], u[7]));
}

// ROWS sums over the LPH lanes of a head, each of which ends up with one of them (row_lane(i) with that of row i): half of the
// rows' shares go to the other half of the lanes, and so on, so that each lane's share is added once.
template <int ROWS, int LPH>
__device__ __forceinline__ constexpr int row_lane(int i) {
  return ROWS == 1 ? 0 : ROWS <= 4 ? (i >> 1 & 1) * (LPH / 2) + (i & 1) * (LPH / 4) : (i >> 2 & 1) * (LPH / 2) + (i >> 1 & 1) * (LPH / 4) + (i & 1) * (LPH / 8);
}
template <int ROWS, int LPH>
__device__ __forceinline__ double sum_rows(const double (&s)[ROWS], int lane) {
  constexpr int P = ROWS == 1 ? 1 : ROWS <= 4 ? 4 : 8;
  static_assert(ROWS <= 8 && P <= LPH, "a lane to a row");
  double v[P];
#pragma unroll
  for (int i = 0; i < P; ++i) v[i] = i < ROWS ? s[i < ROWS ? i : 0] : 0.0;
  int o = LPH / 2;
#pragma unroll
  for (int n = P / 2; n > 0; n >>= 1, o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const double mine = up ? v[i + n] : v[i], give = up ? v[i] : v[i + n];
      v[i] = mine + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
  for (; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
  return v[0];
}
// 8 elements times their gains, from element d on.
__device__ __forceinline__ void scale8(float (&x)[8], const void* gain, int bf16, int d) {
  float g[8];
  load_gain(gain, bf16, d, g);
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float2 y = mul2(make_float2(x[e], x[e + 1]), make_float2(g[e], g[e + 1]));
    x[e] = y.x;
    x[e + 1] = y.y;
  }
}

struct AppendParams {
  KvView c;
  BatchView b;
  const __nv_bfloat16 *k, *v, *q;
  __nv_bfloat16* q_out;
  long k_ts, k_hs, v_ts, v_hs, q_ts, q_hs, qo_ts, qo_hs;
  const float4* table;
  const int32_t* positions;
  int* status;
  int n_heads, n_pos, rot_dim, blocks_per_token, groups;       // n_heads 0: no queries; groups: heads side by side in a block
  float eps;
};
// (Apart: with these in AppendParams every append takes 0.3 us longer to launch.)
struct AppendNormParams : AppendParams {
  const void *q_gain, *k_gain;                                 // hbl_kv_append_norm; NULL: ones
  int gain_bf16;
  float norm_eps;
};
template <bool NORM> struct ParamsOf { using type = AppendParams; };
template <> struct ParamsOf<true> { using type = AppendNormParams; };

// Where a token goes: the block's token t, looked up by every warp for itself.  False: nowhere (reported, or behind the
// last sequence).
struct Place { int b, pos, page, slot, slot8; };             // slot8: row of the 8-bit first tokens, -1: none
template <bool BOS>
__device__ __forceinline__ bool find_place(const KvView& c, const BatchView& s, int t, int lane, int* status, Place& o) {
  o.b = find_sequence(s.q_start, s.n_seqs, t, lane);
  if (o.b >= s.n_seqs) return false;                          // a row behind the last sequence
  SeqLens len;
  if (!sequence_lengths(s, o.b, c.page_shift, status, len)) return false;
  const long place = (long)len.kv - len.q_len + (t - len.q0);
  o.pos = (int)place;
  o.slot8 = -1;
  bool good = place >= 0 && place < len.held && t >= len.q0;
  if (good) {
    o.page = __ldg(s.pages + (long)o.b * s.max_pages + (place >> c.page_shift));
    o.slot = (int)place & ((1 << c.page_shift) - 1);
    good = o.page >= 0 && o.page < c.n_pages;
    if (BOS && good && place == 0 && c.bos_k != nullptr) {
      o.slot8 = s.bos_slot != nullptr ? __ldg(s.bos_slot + o.b) : o.b;
      good = o.slot8 >= 0 && o.slot8 < c.n_slots;
    }
  }
  if (!good) report_device_error(status, HBL_ERR_RANGE);
  return good;
}

// BITS 3, 4, 8 or 16; LPH = head_dim / 8 lanes to a head; a thread takes ROWS heads (queries, then keys, then
// values) of one token.  A thread block works on one token.  EVEN: the numbers of heads are multiples of a warp's, so all
// of a warp's heads are queries, or keys, or values, and what depends on that is decided once for the warp.
// (Four 2048-token prompts of 96 heads: 8 bits 153 us without, 132 with it, bf16 81 and 72, 3 bits 151 and 148.)
// Six heads to a thread at 3 and 4 bits: kept to 64 registers (4 bits 137 us; 171 with the 96 that it would take).
// NORM: queries and keys are r R(gain x), r = 1 / sqrt(mean x^2 + eps).  R is linear, so r goes last; x's squares are summed in fp64
// (a bf16 value's is exact) and r is rounded once, so that a key's codes are those of the fp32 formula, bit for bit.
template <int BITS, int LPH, bool INTERLEAVED, int ROWS, bool EVEN, bool NORM>
__global__ void __launch_bounds__(kThreads, ROWS >= 4 && (NORM || (ROWS == 6 && BITS < 8)) ? 4 : 0) kv_append_kernel(const __grid_constant__ typename ParamsOf<NORM>::type p) {
  constexpr int HPW = 32 / LPH;                               // heads side by side in a warp
  const int groups = p.groups;                                // ... and in the block
  grid_dependency_wait();
  const int t = blockIdx.x / p.blocks_per_token, part = blockIdx.x % p.blocks_per_token;
  const bool there = t < __ldg(p.b.q_start + p.b.n_seqs);     // behind the last sequence the tensors need not have the row
  const int lane = threadIdx.x & 31, j = threadIdx.x % LPH, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  const int kvh = p.c.n_kv_heads, first_v = p.n_heads + kvh, rows = first_v + kvh;
  const __nv_bfloat16 *q = p.q + t * p.q_ts, *k = p.k + t * p.k_ts, *v = p.v + t * p.v_ts;
  const int first = part * (ROWS * groups) + warp * HPW;      // the warp's rows: first + i * groups + 0 .. HPW - 1
  const int own = lane / LPH;                                 // which of them is the thread's
  // A row's number, as far as what it is goes by it; what is left of the thread's own is a multiple of the head's stride.
  const int r0 = EVEN ? first : first + own, rest = EVEN ? own : 0;
  uint4 raw[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int r = r0 + i * groups;
    raw[i] = make_uint4(0, 0, 0, 0);
    if (there && r < rows) {
      const long hs = r < p.n_heads ? p.q_hs : r < first_v ? p.k_hs : p.v_hs;
      const __nv_bfloat16* src = r < p.n_heads ? q + r * hs : r < first_v ? k + (r - p.n_heads) * hs : v + (r - first_v) * hs;
      raw[i] = *reinterpret_cast<const uint4*>(src + rest * hs + 8 * j);
    }
  }
  Place at;
  if (!find_place<(BITS < 8)>(p.c, p.b, t, lane, p.status, at) || !there) return;
  const int turn = p.positions != nullptr ? __ldg(p.positions + t) : at.pos;
  if (p.table != nullptr && (turn < 0 || turn >= p.n_pos)) {
    report_device_error(p.status, HBL_ERR_RANGE);
    return;
  }
  // ---- the lane's pairs: 4 of the interleaved layout, 8 of the half layout (elements 8j .. 8j + 7 and their partners).
  // Lower half: c x1 - s x2; upper half: c x2 + s x1: the sign goes into s, products and sum are rounded one by one. ----
  constexpr int PAIRS = INTERLEAVED ? 4 : 8;
  const int half8 = p.rot_dim / 16;                           // lanes to half of the rotated part
  const bool turned = p.table != nullptr && 8 * j < p.rot_dim;
  const bool upper = !INTERLEAVED && j >= half8;
  const int partner = (lane & ~(LPH - 1)) + (turned ? (upper ? j - half8 : j + half8) : j);
  float c[PAIRS], s[PAIRS];
  if (turned) {
    const int first = INTERLEAVED ? 4 * j : 8 * (upper ? j - half8 : j);
    const float4* row = p.table + ((long)turn * (p.rot_dim / 2) + first) / 2;
#pragma unroll
    for (int i = 0; i < PAIRS / 2; ++i) {
      const float4 x = __ldg(row + i);
      c[2 * i] = x.x; s[2 * i] = upper ? x.y : -x.y; c[2 * i + 1] = x.z; s[2 * i + 1] = upper ? x.w : -x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) { c[i] = 1.f; s[i] = 0.f; }
  }
  float root = 1.f;                                            // NORM: of the lane's row, see row_lane
  if constexpr (NORM) {
    double sum[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      sum[i] = 0.0;
      if (EVEN && r0 + i * groups >= first_v) continue;
      float x[8];
      widen8(raw[i], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[i] = fma((double)x[e], (double)x[e], sum[i]);
    }
    root = inverse_root(fma(sum_rows<ROWS, LPH>(sum, lane), 1.0 / (8 * LPH), (double)p.norm_eps));
  }
  const long row0 = cache_row(p.c, at.page, 0, at.slot);      // head h: row0 + (h << page_shift)
  float f[BITS == 16 ? 1 : ROWS][8];
  uint32_t top[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int r = r0 + i * groups;
    float (&x)[8] = f[BITS == 16 ? 0 : i];
    top[i] = 0;
    widen8(raw[i], x);
    const float inv = NORM ? __shfl_sync(0xffffffffu, root, (lane & ~(LPH - 1)) + row_lane<ROWS, LPH>(i)) : 1.f;
    if constexpr (NORM) {
      const void* gain = r < p.n_heads ? p.q_gain : r < first_v ? p.k_gain : nullptr;
      if (gain != nullptr) scale8(x, gain, p.gain_bf16, 8 * j);
    }
    const bool rotate = turned && r < first_v;
    if (EVEN ? p.table != nullptr && r < first_v : __any_sync(0xffffffffu, rotate)) {      // (the whole warp: it shuffles)
      if constexpr (!INTERLEAVED) {
        float g[8];
        if constexpr (NORM) {                                  // (with its gain: eight shuffles, against four, the gain and its product)
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = __shfl_sync(0xffffffffu, x[e], partner);
        } else {
          uint4 other;
          other.x = __shfl_sync(0xffffffffu, raw[i].x, partner);
          other.y = __shfl_sync(0xffffffffu, raw[i].y, partner);
          other.z = __shfl_sync(0xffffffffu, raw[i].z, partner);
          other.w = __shfl_sync(0xffffffffu, raw[i].w, partner);
          widen8(other, g);
        }
        if (rotate) {
          // (packed products: 3-bit prompts 185 -> 181 us with the norm, but 148 -> 152 without)
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            float2 own = make_float2(x[e], x[e + 1]), its = make_float2(g[e], g[e + 1]);
            const float2 cs = make_float2(c[e], c[e + 1]), sn = make_float2(s[e], s[e + 1]);
            if constexpr (NORM) {
              own = mul2(own, cs);
              its = mul2(its, sn);
            } else {
              own = make_float2(__fmul_rn(own.x, cs.x), __fmul_rn(own.y, cs.y));
              its = make_float2(__fmul_rn(its.x, sn.x), __fmul_rn(its.y, sn.y));
            }
            x[e] = __fadd_rn(own.x, its.x);
            x[e + 1] = __fadd_rn(own.y, its.y);
          }
        }
      } else if (rotate) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x1 = x[2 * e], x2 = x[2 * e + 1];
          x[2 * e] = __fadd_rn(__fmul_rn(x1, c[e]), __fmul_rn(x2, s[e]));
          x[2 * e + 1] = __fsub_rn(__fmul_rn(x2, c[e]), __fmul_rn(x1, s[e]));
        }
      }
    }
    if (NORM && r < first_v) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float2 y = mul2(make_float2(x[e], x[e + 1]), make_float2(inv, inv));
        x[e] = y.x;
        x[e + 1] = y.y;
      }
    }
    if (r < p.n_heads) {
      *reinterpret_cast<uint4*>(p.q_out + t * p.qo_ts + r * p.qo_hs + (rest * p.qo_hs + 8 * j)) = narrow8(x);
    } else if (BITS == 16 && r < rows) {
      const bool key = r < first_v;
      const long row = row0 + ((long)(r - (key ? p.n_heads : first_v) + rest) << p.c.page_shift);
      *reinterpret_cast<uint4*>((key ? p.c.k : p.c.v) + (row * LPH + j) * 16) = narrow8(x);
    }
    if (BITS < 16 && !(EVEN && r < p.n_heads)) {
      // the head's largest magnitude, on the bit patterns: a NaN is larger than everything and is not lost
#pragma unroll
      for (int e = 0; e < 8; ++e) top[i] = max(top[i], __float_as_uint(x[e]) & 0x7FFFFFFFu);
    }
  }
  if constexpr (BITS < 16) {
    if (first + (ROWS - 1) * groups + HPW - 1 < p.n_heads) return;     // (uniform: the warp has queries only)
    constexpr float C = (float)((1 << (BITS - 1)) - 1);
    // Both divisions of a head cost what they cost for a whole warp, so the warp's ROWS * HPW heads are put one to a lane
    // and divided together.
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      if (EVEN && first + i * groups < p.n_heads) continue;
#pragma unroll
      for (int o = LPH / 2; o > 0; o >>= 1) top[i] = max(top[i], __shfl_xor_sync(0xffffffffu, top[i], o));
      const uint32_t x = __shfl_sync(0xffffffffu, top[i], (lane % HPW) * LPH);
      if (lane / HPW == i) mine = x;
    }
    const bool finite = mine < 0x7F800000u;
    const float gamma = finite ? __uint_as_float(mine) : 0.f;
    const float rq_mine = finite ? __fdiv_rn(C, __fadd_rn(gamma, p.eps)) : 0.f;
    if (lane < ROWS * HPW) {
      const int r = first + lane % HPW + (lane / HPW) * groups;                      // this lane's head
      if (r >= p.n_heads && r < rows) {
        const bool key = r < first_v;
        const long row = row0 + ((long)(r - (key ? p.n_heads : first_v)) << p.c.page_shift);
        (key ? p.c.k_scale : p.c.v_scale)[row] = finite ? __fdiv_rn(gamma, C) : __uint_as_float(0x7FC00000u);
      }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int r = r0 + i * groups;
      if (EVEN && (r < p.n_heads || r >= rows)) continue;
      const float rq = __shfl_sync(0xffffffffu, rq_mine, i * HPW + own);
      float (&x)[8] = f[BITS == 16 ? 0 : i];
      if (top[i] >= 0x7F800000u) {                             // the head reads as NaN: its codes are those of zero
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
      }
      const bool store = r >= p.n_heads && r < rows;
      const bool key = r < first_v;
      const int head = r - (key ? p.n_heads : first_v) + rest;
      const long row = row0 + ((long)head << p.c.page_shift);
      const uint2 u = codes8<BITS>(x, rq);
      unsigned char* dst = (key ? p.c.k : p.c.v) + row * (LPH * BITS);
      if constexpr (BITS == 8) {
        if (store) *reinterpret_cast<uint2*>(dst + 8 * j) = u;
      } else if constexpr (BITS == 4) {
        if (store) *reinterpret_cast<uint32_t*>(dst + 4 * j) = __byte_perm(u.x | (u.x >> 4), u.y | (u.y >> 4), 0x6420);
      } else {
        // 24 bits a lane (four codes: bits 0-2, 8-10, .. moved together); four neighbouring lanes make three 32-bit words
        auto twelve = [](uint32_t y) { y = (y & 0x00070007u) | ((y >> 5) & 0x00380038u); return (y & 0x3Fu) | ((y >> 10) & 0xFC0u); };
        const uint32_t o = twelve(u.x) | twelve(u.y) << 12;
        const uint32_t next = __shfl_down_sync(0xffffffffu, o, 1);
        const int w = j & 3;
        const uint32_t word = w == 0 ? (o | (next << 24)) : w == 1 ? ((o >> 8) | (next << 16)) : ((o >> 16) | (next << 8));
        if (store && w < 3) *reinterpret_cast<uint32_t*>(dst + 12 * (j >> 2) + 4 * w) = word;
      }
      if (BITS < 8 && store && at.slot8 >= 0) {                // the sequence's first token, at 8 bits as well
        const bool sane = top[i] < 0x7F800000u;
        const float g = __uint_as_float(top[i]);
        const long brow = (long)at.slot8 * kvh + head;
        const float rq8 = sane ? __fdiv_rn(127.0f, __fadd_rn(g, p.eps)) : 0.f;
        *reinterpret_cast<uint2*>((key ? p.c.bos_k : p.c.bos_v) + (brow * LPH + j) * 8) = codes8<8>(x, rq8);
        if (j == 0) (key ? p.c.bos_k_scale : p.c.bos_v_scale)[brow] = sane ? __fdiv_rn(g, 127.0f) : __uint_as_float(0x7FC00000u);
      }
    }
  }
}

struct ReadParams {
  KvView c;
  BatchView b;
  uint4 *k_out, *v_out;
  int* status;
  int blocks_per_token, groups;
};

// A thread takes ROWS heads (keys, then values) of one token; a thread block works on one token.
template <int BITS, int LPH, int ROWS>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const __grid_constant__ ReadParams p) {
  grid_dependency_wait();
  const int t = blockIdx.x / p.blocks_per_token, part = blockIdx.x % p.blocks_per_token;
  const int lane = threadIdx.x & 31, j = threadIdx.x % LPH, group = threadIdx.x / LPH, kvh = p.c.n_kv_heads;
  Place at;
  if (!find_place<(BITS < 8)>(p.c, p.b, t, lane, p.status, at)) return;
  const long row0 = cache_row(p.c, at.page, 0, at.slot);
  uint2 u[ROWS];
  uint4 whole[ROWS];
  float scale[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int r = (part * ROWS + i) * p.groups + group;
    u[i] = make_uint2(0, 0);
    whole[i] = make_uint4(0, 0, 0, 0);
    scale[i] = 0.f;
    if (r >= 2 * kvh) continue;
    const bool key = r < kvh;
    const int head = key ? r : r - kvh;
    const long row = row0 + ((long)head << p.c.page_shift);
    const unsigned char* base = key ? p.c.k : p.c.v;
    if (BITS == 16) {
      whole[i] = *reinterpret_cast<const uint4*>(base + (row * LPH + j) * 16);
    } else if (BITS == 8 || at.slot8 >= 0) {
      const long brow = (long)at.slot8 * kvh + head;
      u[i] = *(reinterpret_cast<const uint2*>(BITS < 8 ? (key ? p.c.bos_k : p.c.bos_v) + brow * LPH * 8 : base + row * LPH * 8) + j);
      scale[i] = BITS < 8 ? (key ? p.c.bos_k_scale : p.c.bos_v_scale)[brow] : (key ? p.c.k_scale : p.c.v_scale)[row];
    } else {
      scale[i] = (key ? p.c.k_scale : p.c.v_scale)[row];
      if (BITS == 4) {
        u[i].x = *reinterpret_cast<const uint32_t*>(base + (row * LPH + j) * 4);
      } else {                                                 // 24 bits, anywhere in a word or across two of the row
        const uint32_t* w = reinterpret_cast<const uint32_t*>(base + row * (LPH * 3)) + (3 * j >> 2);
        u[i] = make_uint2(w[0], w[(3 * j & 3) > 1 ? 1 : 0]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int r = (part * ROWS + i) * p.groups + group;
    if (r >= 2 * kvh) continue;
    uint4 o = whole[i];
    if constexpr (BITS < 16) {
      float x[8];
      if (BITS == 8 || at.slot8 >= 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)((int)(((e < 4 ? u[i].x : u[i].y) >> (8 * (e & 3))) & 255u) - 128);
      } else {
        const uint32_t bits = BITS == 4 ? u[i].x : __funnelshift_r(u[i].x, u[i].y, (3 * j & 3) * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)((int)((bits >> (BITS * e)) & ((1u << BITS) - 1)) - (1 << (BITS - 1)));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= scale[i];
      o = narrow8(x);
    }
    (r < kvh ? p.k_out : p.v_out)[((long)t * kvh + (r < kvh ? r : r - kvh)) * LPH + j] = o;
  }
}

// Blocks to a token and heads side by side in a block, so that as few as can be of a token's places stay empty.  (Blocks of
// 256 threads whatever the heads: sixteen 2048-token prompts of 16 and 2 heads 232 us instead of 106.)
struct Deal { int blocks, groups; };
Deal deal(int rows, int lph, int rows_per_thread) {
  const int most = kThreads / lph, warp = 32 / lph;
  Deal d;
  d.blocks = (rows + rows_per_thread * most - 1) / (rows_per_thread * most);
  const int need = (rows + rows_per_thread * d.blocks - 1) / (rows_per_thread * d.blocks);
  d.groups = (need + warp - 1) / warp * warp;
  return d;
}
template <int BITS, int LPH, bool INTERLEAVED, int ROWS, bool EVEN, bool NORM>
int launch_append_rows(typename ParamsOf<NORM>::type& p, cudaStream_t s) {
  const Deal d = deal(p.n_heads + 2 * p.c.n_kv_heads, LPH, ROWS);
  p.blocks_per_token = d.blocks;
  p.groups = d.groups;
  const long blocks = (long)p.b.tokens * d.blocks;
  if (blocks > 0x7fffffffL) return HBL_ERR_TOO_LARGE;
  HBL_CUDA_OK(launch_waiting(kv_append_kernel<BITS, LPH, INTERLEAVED, ROWS, EVEN, NORM>, dim3((unsigned)blocks), dim3(d.groups * LPH), 0, s, p));
  note_launch();
  return HBL_OK;
}
// One head to a thread for a decoding step, whose latency counts.  Where the call fills the GPU six (four 2048-token prompts
// of 96 heads at 3 bits: 148 us; four or three heads 163, two 180; 48 heads 64, 71, 70, 75), or four at head_dim 256, where six
// run out of registers (341 us against 291).
template <int BITS, int LPH, bool INTERLEAVED, bool EVEN, bool NORM>
int launch_append_layout(typename ParamsOf<NORM>::type& p, cudaStream_t s) {
  if ((long)p.b.tokens * (p.n_heads + 2 * p.c.n_kv_heads) * LPH < (long)sm_count() * 2048 * 4)
    return launch_append_rows<BITS, LPH, INTERLEAVED, 1, EVEN, NORM>(p, s);
  return launch_append_rows<BITS, LPH, INTERLEAVED, LPH < 32 ? 6 : 4, EVEN, NORM>(p, s);
}
template <int BITS, int LPH, bool NORM>
int launch_append_heads(typename ParamsOf<NORM>::type& p, bool interleaved, cudaStream_t s) {
  if ((p.n_heads | p.c.n_kv_heads) % (32 / LPH) == 0)
    return interleaved ? launch_append_layout<BITS, LPH, true, true, NORM>(p, s) : launch_append_layout<BITS, LPH, false, true, NORM>(p, s);
  return interleaved ? launch_append_layout<BITS, LPH, true, false, NORM>(p, s) : launch_append_layout<BITS, LPH, false, false, NORM>(p, s);
}
template <int BITS, bool NORM>
int launch_append_dim(typename ParamsOf<NORM>::type& p, bool interleaved, cudaStream_t s) {
  switch (p.c.head_dim) {
    case 64: return launch_append_heads<BITS, 8, NORM>(p, interleaved, s);
    case 128: return launch_append_heads<BITS, 16, NORM>(p, interleaved, s);
    case 256: return launch_append_heads<BITS, 32, NORM>(p, interleaved, s);
    default: return HBL_ERR_SHAPE;
  }
}
template <int BITS>
int launch_append_bits(AppendNormParams& p, bool interleaved, bool norm, cudaStream_t s) {
  return norm ? launch_append_dim<BITS, true>(p, interleaved, s) : launch_append_dim<BITS, false>(static_cast<AppendParams&>(p), interleaved, s);
}

template <int BITS, int LPH, int ROWS>
int launch_read_rows(ReadParams& p, cudaStream_t s) {
  const Deal d = deal(2 * p.c.n_kv_heads, LPH, ROWS);
  p.blocks_per_token = d.blocks;
  p.groups = d.groups;
  const long blocks = (long)p.b.tokens * d.blocks;
  if (blocks > 0x7fffffffL) return HBL_ERR_TOO_LARGE;
  HBL_CUDA_OK(launch_waiting(kv_read_kernel<BITS, LPH, ROWS>, dim3((unsigned)blocks), dim3(d.groups * LPH), 0, s, p));
  note_launch();
  return HBL_OK;
}
template <int BITS, int LPH>
int launch_read_one(ReadParams& p, cudaStream_t s) {
  const long threads = (long)p.b.tokens * 2 * p.c.n_kv_heads * LPH;
  if (threads >= (long)sm_count() * 2048 * 4) return launch_read_rows<BITS, LPH, 4>(p, s);
  return launch_read_rows<BITS, LPH, 1>(p, s);
}
template <int BITS>
int launch_read_bits(ReadParams& p, cudaStream_t s) {
  switch (p.c.head_dim) {
    case 64: return launch_read_one<BITS, 8>(p, s);
    case 128: return launch_read_one<BITS, 16>(p, s);
    case 256: return launch_read_one<BITS, 32>(p, s);
    default: return HBL_ERR_SHAPE;
  }
}

}  // namespace

int launch_kv_append(const KvView& c, const BatchView& b, const hbl_kv_append_t& a, const hbl_head_norm_t* norm, cudaStream_t s) {
  AppendNormParams p{};
  p.c = c; p.b = b;
  p.k = static_cast<const __nv_bfloat16*>(a.k); p.v = static_cast<const __nv_bfloat16*>(a.v);
  p.q = static_cast<const __nv_bfloat16*>(a.q); p.q_out = static_cast<__nv_bfloat16*>(a.q_out);
  p.k_ts = a.k_token_stride; p.k_hs = a.k_head_stride; p.v_ts = a.v_token_stride; p.v_hs = a.v_head_stride;
  p.q_ts = a.q_token_stride; p.q_hs = a.q_head_stride; p.qo_ts = a.q_out_token_stride; p.qo_hs = a.q_out_head_stride;
  p.table = reinterpret_cast<const float4*>(a.table); p.positions = a.positions;
  p.n_heads = a.q != nullptr ? a.n_heads : 0;
  p.n_pos = a.n_pos; p.rot_dim = a.table != nullptr ? a.rot_dim : 0; p.eps = a.eps;
  p.status = device_status_word();
  if (p.status == nullptr) return HBL_ERR_CUDA;
  if (norm != nullptr) {
    p.q_gain = norm->q_gain; p.k_gain = norm->k_gain; p.gain_bf16 = norm->gain_dtype == HBL_BF16; p.norm_eps = norm->norm_eps;
  }
  const bool inter = a.layout == HBL_ROPE_INTERLEAVED;
  switch (c.bits) {
    case 3: return launch_append_bits<3>(p, inter, norm != nullptr, s);
    case 4: return launch_append_bits<4>(p, inter, norm != nullptr, s);
    case 8: return launch_append_bits<8>(p, inter, norm != nullptr, s);
    case 16: return launch_append_bits<16>(p, inter, norm != nullptr, s);
    default: return HBL_ERR_BITS;
  }
}

int launch_kv_read(const KvView& c, const BatchView& b, void* k_out, void* v_out, cudaStream_t s) {
  ReadParams p{};
  p.c = c; p.b = b;
  p.k_out = static_cast<uint4*>(k_out); p.v_out = static_cast<uint4*>(v_out);
  p.status = device_status_word();
  if (p.status == nullptr) return HBL_ERR_CUDA;
  switch (c.bits) {
    case 3: return launch_read_bits<3>(p, s);
    case 4: return launch_read_bits<4>(p, s);
    case 8: return launch_read_bits<8>(p, s);
    case 16: return launch_read_bits<16>(p, s);
    default: return HBL_ERR_BITS;
  }
}

}  // namespace hbl
