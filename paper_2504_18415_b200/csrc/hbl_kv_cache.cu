// The paged cache of attention states: tokens into it (keys rotated, keys and values quantized per head, queries
// rotated, all in one launch) and out of it as bf16 values.
//
//   gamma = max_d |x[d]|,  u = round((2^(b-1) - 1) / (gamma + eps) * x) + 2^(b-1),  scale = gamma / (2^(b-1) - 1)
//
// Bound by HBM for prompts (2 bytes read and b / 8 written per element, queries 2 and 2) and by the chain of dependent
// loads (sequence -> length -> page -> row) for a decoding step.  A lane owns 8 consecutive elements of a head, so a head
// is head_dim / 8 lanes and its maximum takes three to five shuffles; the partner of a rotated element lies in the same
// lane (interleaved layout) or one shuffle away (half layout).  A thread takes ROWS heads of the same token: the table's
// pairs are loaded once for all of them, and their loads are in flight together.  The loads of the data do not depend on
// that chain and are issued before it.
#include "hbl_kv_cache.cuh"

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

struct AppendParams {
  KvView c;
  BatchView b;
  const __nv_bfloat16 *k, *v, *q;
  __nv_bfloat16* q_out;
  long k_ts, k_hs, v_ts, v_hs, q_ts, q_hs, qo_ts, qo_hs;
  const float4* table;
  const int32_t* positions;
  int* status;
  int n_heads, n_pos, rot_dim, blocks_per_token;               // n_heads 0: no queries
  float eps;
};

// BITS 3, 4, 8 or 16; LPH = head_dim / 8 lanes to a head; a thread takes ROWS heads (queries, then keys, then
// values) of one token.  A thread block works on one token.
template <int BITS, int LPH, bool INTERLEAVED, int ROWS>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int GROUPS = kThreads / LPH;                      // heads side by side in the block
  grid_dependency_wait();
  const int t = blockIdx.x / p.blocks_per_token, part = blockIdx.x % p.blocks_per_token;
  const int lane = threadIdx.x & 31, j = threadIdx.x % LPH, group = threadIdx.x / LPH;
  const int kvh = p.c.n_kv_heads, rows = p.n_heads + 2 * kvh;
  uint4 raw[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int r = (part * ROWS + i) * GROUPS + group;
    raw[i] = make_uint4(0, 0, 0, 0);
    if (r < rows) {
      const __nv_bfloat16* src = r < p.n_heads         ? p.q + t * p.q_ts + r * p.q_hs
                                 : r < p.n_heads + kvh ? p.k + t * p.k_ts + (r - p.n_heads) * p.k_hs
                                                       : p.v + t * p.v_ts + (r - p.n_heads - kvh) * p.v_hs;
      raw[i] = *reinterpret_cast<const uint4*>(src + 8 * j);
    }
  }
  // ---- where the token goes ----
  const int b = find_sequence(p.b.q_start, p.b.n_seqs, t, lane);
  if (b >= p.b.n_seqs) return;                                // a row behind the last sequence
  SeqLens len;
  if (!sequence_lengths(p.b, b, p.c.page_shift, p.status, len)) return;
  const long place = (long)len.kv - len.q_len + (t - len.q0);
  bool good = place >= 0 && place < len.held && t >= len.q0;
  const int at = p.positions != nullptr ? __ldg(p.positions + t) : (int)place;
  int page = 0, slot8 = -1;
  if (good) {
    page = __ldg(p.b.pages + (long)b * p.b.max_pages + (place >> p.c.page_shift));
    good = page >= 0 && page < p.c.n_pages && (p.table == nullptr || (at >= 0 && at < p.n_pos));
    if (good && place == 0 && p.c.bos_k != nullptr) {
      slot8 = p.b.bos_slot != nullptr ? __ldg(p.b.bos_slot + b) : b;
      good = slot8 >= 0 && slot8 < p.c.n_slots;
    }
  }
  if (!good) {
    report_device_error(p.status, HBL_ERR_RANGE);
    return;
  }
  // ---- the lane's pairs: 4 of the interleaved layout, 8 of the half layout (elements 8j .. 8j + 7 and their partners) ----
  constexpr int PAIRS = INTERLEAVED ? 4 : 8;
  const int half8 = p.rot_dim / 16;                           // lanes to half of the rotated part
  const bool turned = p.table != nullptr && 8 * j < p.rot_dim;
  const bool upper = !INTERLEAVED && j >= half8;
  const int partner = (lane & ~(LPH - 1)) + (turned ? (upper ? j - half8 : j + half8) : j);
  float c[PAIRS], s[PAIRS];
  if (turned) {
    const int first = INTERLEAVED ? 4 * j : 8 * (upper ? j - half8 : j);
    const float4* row = p.table + ((long)at * (p.rot_dim / 2) + first) / 2;
#pragma unroll
    for (int i = 0; i < PAIRS / 2; ++i) {
      const float4 v = __ldg(row + i);
      c[2 * i] = v.x; s[2 * i] = v.y; c[2 * i + 1] = v.z; s[2 * i + 1] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) { c[i] = 1.f; s[i] = 0.f; }
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int r = (part * ROWS + i) * GROUPS + group;
    const int kind = r < p.n_heads ? 0 : r < p.n_heads + kvh ? 1 : 2;
    float f[8];
    widen8(raw[i], f);
    // (every lane of the warp takes part in the shuffles, whatever its rows are)
    if constexpr (!INTERLEAVED) {
      uint4 other;
      other.x = __shfl_sync(0xffffffffu, raw[i].x, partner);
      other.y = __shfl_sync(0xffffffffu, raw[i].y, partner);
      other.z = __shfl_sync(0xffffffffu, raw[i].z, partner);
      other.w = __shfl_sync(0xffffffffu, raw[i].w, partner);
      if (turned && kind != 2) {
        float g[8];
        widen8(other, g);
#pragma unroll
        for (int k = 0; k < 8; ++k)                            // lower half: c x1 - s x2; upper half: c x2 + s x1
          f[k] = upper ? __fadd_rn(__fmul_rn(f[k], c[k]), __fmul_rn(g[k], s[k]))
                       : __fsub_rn(__fmul_rn(f[k], c[k]), __fmul_rn(g[k], s[k]));
      }
    } else if (turned && kind != 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x1 = f[2 * k], x2 = f[2 * k + 1];
        f[2 * k] = __fsub_rn(__fmul_rn(x1, c[k]), __fmul_rn(x2, s[k]));
        f[2 * k + 1] = __fadd_rn(__fmul_rn(x2, c[k]), __fmul_rn(x1, s[k]));
      }
    }
    const int head = kind == 1 ? r - p.n_heads : r - p.n_heads - kvh;
    const bool live = r < rows;
    if (kind == 0 && live) *reinterpret_cast<uint4*>(p.q_out + t * p.qo_ts + r * p.qo_hs + 8 * j) = narrow8(f);
    const bool store = live && kind != 0;
    const long row = store ? cache_row(p.c, page, head, (int)(place & ((1 << p.c.page_shift) - 1))) : 0;
    unsigned char* base = kind == 1 ? p.c.k : p.c.v;
    if constexpr (BITS == 16) {
      if (store) *reinterpret_cast<uint4*>(base + (row * LPH + j) * 16) = narrow8(f);
    } else {
      // the head's largest magnitude, on the bit patterns: a NaN is larger than everything and is not lost
      uint32_t m = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) m = max(m, __float_as_uint(f[k]) & 0x7FFFFFFFu);
#pragma unroll
      for (int o = LPH / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      const bool finite = m < 0x7F800000u;
      const float gamma = __uint_as_float(m);
      constexpr float C = (float)((1 << (BITS - 1)) - 1);
      const float rq = finite ? __fdiv_rn(C, __fadd_rn(gamma, p.eps)) : 0.f;
      const float scale = finite ? __fdiv_rn(gamma, C) : __uint_as_float(0x7FC00000u);
      if (!finite) {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = 0.f;
      }
      const uint2 u = codes8<BITS>(f, rq);
      unsigned char* dst = base + row * (LPH * BITS);
      if constexpr (BITS == 8) {
        if (store) *reinterpret_cast<uint2*>(dst + 8 * j) = u;
      } else if constexpr (BITS == 4) {
        if (store) *reinterpret_cast<uint32_t*>(dst + 4 * j) = __byte_perm(u.x | (u.x >> 4), u.y | (u.y >> 4), 0x6420);
      } else {
        // 24 bits a lane; four neighbouring lanes make three 32-bit words
        uint32_t o = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) o |= (((u.x >> (8 * k)) & 7u) << (3 * k)) | (((u.y >> (8 * k)) & 7u) << (3 * k + 12));
        const uint32_t next = __shfl_down_sync(0xffffffffu, o, 1);
        const int q = j & 3;
        const uint32_t word = q == 0 ? (o | (next << 24)) : q == 1 ? ((o >> 8) | (next << 16)) : ((o >> 16) | (next << 8));
        if (store && q < 3) *reinterpret_cast<uint32_t*>(dst + 12 * (j >> 2) + 4 * q) = word;
      }
      if (store && j == 0) (kind == 1 ? p.c.k_scale : p.c.v_scale)[row] = scale;
      if (BITS < 8 && store && slot8 >= 0) {                  // the sequence's first token, at 8 bits as well
        const long brow = (long)slot8 * kvh + head;
        const float rq8 = finite ? __fdiv_rn(127.0f, __fadd_rn(gamma, p.eps)) : 0.f;
        *reinterpret_cast<uint2*>((kind == 1 ? p.c.bos_k : p.c.bos_v) + (brow * LPH + j) * 8) = codes8<8>(f, rq8);
        if (j == 0) (kind == 1 ? p.c.bos_k_scale : p.c.bos_v_scale)[brow] = finite ? __fdiv_rn(gamma, 127.0f) : scale;
      }
    }
  }
}

struct ReadParams {
  KvView c;
  BatchView b;
  uint4 *k_out, *v_out;
  int* status;
  int blocks_per_token;
};

template <int BITS, int LPH>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const __grid_constant__ ReadParams p) {
  constexpr int GROUPS = kThreads / LPH;
  grid_dependency_wait();
  const int t = blockIdx.x / p.blocks_per_token, part = blockIdx.x % p.blocks_per_token;
  const int lane = threadIdx.x & 31, j = threadIdx.x % LPH;
  const int b = find_sequence(p.b.q_start, p.b.n_seqs, t, lane);
  if (b >= p.b.n_seqs) return;
  SeqLens len;
  if (!sequence_lengths(p.b, b, p.c.page_shift, p.status, len)) return;
  const int r = part * GROUPS + threadIdx.x / LPH, kvh = p.c.n_kv_heads;
  if (r >= 2 * kvh) return;
  const long place = (long)len.kv - len.q_len + (t - len.q0);
  bool good = place >= 0 && place < len.held && t >= len.q0;
  int page = 0, slot8 = -1;
  if (good) {
    page = __ldg(p.b.pages + (long)b * p.b.max_pages + (place >> p.c.page_shift));
    good = page >= 0 && page < p.c.n_pages;
    if (BITS < 8 && place == 0 && p.c.bos_k != nullptr) {
      slot8 = p.b.bos_slot != nullptr ? __ldg(p.b.bos_slot + b) : b;
      good = good && slot8 >= 0 && slot8 < p.c.n_slots;
    }
  }
  if (!good) {
    report_device_error(p.status, HBL_ERR_RANGE);
    return;
  }
  const bool key = r < kvh;
  const int head = key ? r : r - kvh;
  const long row = cache_row(p.c, page, head, (int)(place & ((1 << p.c.page_shift) - 1)));
  const unsigned char* base = key ? p.c.k : p.c.v;
  uint4 o;
  if constexpr (BITS == 16) {
    o = *reinterpret_cast<const uint4*>(base + (row * LPH + j) * 16);
  } else {
    float f[8];
    float scale = (key ? p.c.k_scale : p.c.v_scale)[row];
    if (slot8 >= 0 || BITS == 8) {
      const long brow = (long)slot8 * kvh + head;
      const unsigned char* src = slot8 >= 0 ? (key ? p.c.bos_k : p.c.bos_v) + brow * LPH * 8 : base + row * LPH * 8;
      if (slot8 >= 0) scale = (key ? p.c.bos_k_scale : p.c.bos_v_scale)[brow];
      const uint2 u = *reinterpret_cast<const uint2*>(src + 8 * j);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = (float)((int)(((k < 4 ? u.x : u.y) >> (8 * (k & 3))) & 255u) - 128);
    } else if constexpr (BITS == 4) {
      const uint32_t u = *reinterpret_cast<const uint32_t*>(base + (row * LPH + j) * 4);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = (float)((int)((u >> (4 * k)) & 15u) - 8);
    } else {
      const unsigned char* src = base + (row * LPH + j) * 3;
      const uint32_t u = src[0] | ((uint32_t)src[1] << 8) | ((uint32_t)src[2] << 16);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = (float)((int)((u >> (3 * k)) & 7u) - 4);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] *= scale;
    o = narrow8(f);
  }
  (key ? p.k_out : p.v_out)[((long)t * kvh + head) * LPH + j] = o;
}

template <int BITS, int LPH, bool INTERLEAVED, int ROWS>
int launch_append_rows(AppendParams& p, cudaStream_t s) {
  const int rows = p.n_heads + 2 * p.c.n_kv_heads, per_block = kThreads / LPH * ROWS;
  p.blocks_per_token = (rows + per_block - 1) / per_block;
  const long blocks = (long)p.b.tokens * p.blocks_per_token;
  if (blocks > 0x7fffffffL) return HBL_ERR_TOO_LARGE;
  HBL_CUDA_OK(launch_dependent(kv_append_kernel<BITS, LPH, INTERLEAVED, ROWS>, dim3((unsigned)blocks), dim3(kThreads), 0, s, p));
  note_launch();
  return HBL_OK;
}
// Four heads to a thread where a decoding step's worth of tokens still fills the GPU, one below.
template <int BITS, int LPH, bool INTERLEAVED>
int launch_append_layout(AppendParams& p, cudaStream_t s) {
  const long threads = (long)p.b.tokens * (p.n_heads + 2 * p.c.n_kv_heads) * LPH;
  if (threads >= (long)sm_count() * 2048 * 4) return launch_append_rows<BITS, LPH, INTERLEAVED, 4>(p, s);
  return launch_append_rows<BITS, LPH, INTERLEAVED, 1>(p, s);
}
template <int BITS>
int launch_append_bits(AppendParams& p, bool interleaved, cudaStream_t s) {
  switch (p.c.head_dim) {
    case 64: return interleaved ? launch_append_layout<BITS, 8, true>(p, s) : launch_append_layout<BITS, 8, false>(p, s);
    case 128: return interleaved ? launch_append_layout<BITS, 16, true>(p, s) : launch_append_layout<BITS, 16, false>(p, s);
    case 256: return interleaved ? launch_append_layout<BITS, 32, true>(p, s) : launch_append_layout<BITS, 32, false>(p, s);
    default: return HBL_ERR_SHAPE;
  }
}

template <int BITS, int LPH>
int launch_read_one(ReadParams& p, cudaStream_t s) {
  const int per_block = kThreads / LPH;
  p.blocks_per_token = (2 * p.c.n_kv_heads + per_block - 1) / per_block;
  const long blocks = (long)p.b.tokens * p.blocks_per_token;
  if (blocks > 0x7fffffffL) return HBL_ERR_TOO_LARGE;
  HBL_CUDA_OK(launch_dependent(kv_read_kernel<BITS, LPH>, dim3((unsigned)blocks), dim3(kThreads), 0, s, p));
  note_launch();
  return HBL_OK;
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

int launch_kv_append(const KvView& c, const BatchView& b, const hbl_kv_append_t& a, cudaStream_t s) {
  AppendParams p{};
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
  const bool inter = a.layout == HBL_ROPE_INTERLEAVED;
  switch (c.bits) {
    case 3: return launch_append_bits<3>(p, inter, s);
    case 4: return launch_append_bits<4>(p, inter, s);
    case 8: return launch_append_bits<8>(p, inter, s);
    case 16: return launch_append_bits<16>(p, inter, s);
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
