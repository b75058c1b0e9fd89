// Rows of the paged cache as operand fragments of mma.m16n8k16 (bf16 x bf16 -> fp32), straight from global memory.
//
// The order of the summed index of a matrix product is free as long as both operands use the same one, and so is the
// order of the result's rows.  Each is chosen here so that a lane's fragments are made of bytes that it can load in one
// piece, and so that codes become bf16 values two at a time:
//   - `unit`: 8 consecutive elements of a row (BITS bytes).  A lane holds N units of a row; L lanes share the row.
//   - a code u of b bits (b <= 4) becomes the bf16 value 128 + u by putting it into the low mantissa bits of 128.0
//     (0x4300); subtracting 128 + 2^(b-1) is exact.  For 8 bits the low seven bits go that way, and the top bit picks
//     what is subtracted (256 or 128).
#pragma once

#include "hbl_kv_cache.cuh"

namespace hbl {
namespace frag {

__device__ __forceinline__ uint32_t bsub2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// (x & mask) | magic as one instruction.  (Left to the compiler it became two, one for each constant: 132 logic
// instructions to 16 keys instead of 68.)
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t magic) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(x), "r"(mask), "r"(magic));
  return r;
}

// N units of one row for lane `idx` of the L lanes that share the row.
template <int BITS, int N, int L>
struct Lane {
  static constexpr int BYTES = N * BITS;                       // per lane and row
  static constexpr int CHUNK = BITS == 3 ? BYTES : (BYTES < 16 ? BYTES : 16);
  static constexpr int UPC = CHUNK / BITS;                     // units to a chunk (BITS == 3: all of them)
  static constexpr int WORDS = BITS == 3 ? (BYTES <= 8 ? 2 : BYTES / 4) : BYTES / 4;
  uint32_t w[WORDS];
  // The unit of the row (0 .. head_dim / 8 - 1) that is the lane's i-th.
  static __device__ __forceinline__ int unit_of(int i, int idx) { return ((i / UPC) * L + idx) * UPC + i % UPC; }
  __device__ __forceinline__ void load(const unsigned char* __restrict__ row, int idx, bool live) {
    if (live) load(row, idx);
    else clear();
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = 0;
  }
  __device__ __forceinline__ void load(const unsigned char* __restrict__ row, int idx) {
    if constexpr (BITS == 3) {
      const uint32_t* r = reinterpret_cast<const uint32_t*>(row);
      if constexpr (BYTES == 3) {                              // one unit, anywhere in its word or across two
        const int at = (3 * idx) >> 2;
        w[0] = __ldg(r + at);
        w[1] = __ldg(r + min(at + 1, 3 * L / 4 - 1));
      } else if constexpr (BYTES == 6) {
        const int at = (6 * idx) >> 2;
        w[0] = __ldg(r + at);
        w[1] = __ldg(r + at + 1);
      } else {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = __ldg(r + idx * WORDS + i);
      }
    } else {
#pragma unroll
      for (int c = 0; c < BYTES / CHUNK; ++c) {
        const unsigned char* p = row + (c * L + idx) * CHUNK;
        if constexpr (CHUNK == 16) {
          const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
          w[4 * c] = v.x; w[4 * c + 1] = v.y; w[4 * c + 2] = v.z; w[4 * c + 3] = v.w;
        } else if constexpr (CHUNK == 8) {
          const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
          w[0] = v.x; w[1] = v.y;
        } else {
          w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
        }
      }
    }
  }
  // BITS == 3: the 24 bits of unit i (what lies above them is not cleared).
  __device__ __forceinline__ uint32_t bits24(int i, int idx) const {
    if constexpr (BYTES == 3) return __funnelshift_r(w[0], w[1], ((3 * idx) & 3) * 8);
    if constexpr (BYTES == 6) {
      const int sh = ((6 * idx) & 3) * 8;                      // 0 or 16
      return i == 0 ? __funnelshift_r(w[0], w[1], sh) : (sh == 0 ? __funnelshift_r(w[0], w[1], 24) : w[1] >> 8);
    }
    const int bit = 24 * i;
    const int a = bit / 32, sh = bit % 32;
    return sh <= 8 ? w[a] >> sh : __funnelshift_r(w[a], w[a + 1 < WORDS ? a + 1 : a], sh);
  }
};

// Element order of the four pairs a unit gives as an operand whose summed index runs along the row: pair j holds the
// unit's elements lo(j) and hi(j).
template <int BITS>
__device__ __forceinline__ constexpr int pair_lo(int j) { return BITS == 16 ? 2 * j : BITS == 8 ? 4 * (j >> 1) + (j & 1) : j; }
template <int BITS>
__device__ __forceinline__ constexpr int pair_hi(int j) { return BITS == 16 ? 2 * j + 1 : BITS == 8 ? pair_lo<8>(j) + 2 : j + 4; }

template <int BITS>
constexpr uint32_t kOffset = BITS == 3 ? 0x43044304u : 0x43084308u;      // 132, 136 as bf16 pairs
__device__ __forceinline__ uint32_t from_bytes(uint32_t x) {               // bytes 0 and 2: code - 128
  return bsub2(and_or(x, 0x007F007Fu, 0x43004300u), and_or(~x, 0x00800080u, 0x43004300u));
}

// Unit i of a lane as four pairs along the row.
template <int BITS, int N, int L>
__device__ __forceinline__ void pairs(const Lane<BITS, N, L>& r, int i, int idx, uint32_t (&o)[4]) {
  if constexpr (BITS == 16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = r.w[4 * i + j];
  } else if constexpr (BITS == 8) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      o[2 * h] = from_bytes(r.w[2 * i + h]);
      o[2 * h + 1] = from_bytes(r.w[2 * i + h] >> 8);
    }
  } else if constexpr (BITS == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = bsub2(and_or(r.w[i] >> (4 * j), 0x000F000Fu, 0x43004300u), kOffset<4>);
  } else {
    const uint32_t v = r.bits24(i, idx);
    const uint32_t x = (v & 0xFFFu) | ((v << 4) & 0x0FFF0000u);
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = bsub2(and_or(x >> (3 * j), 0x00070007u, 0x43004300u), kOffset<3>);
  }
}
// ---- the same codes as fp16 values: 10 mantissa bits take a code at several places of a word without a shift ----
// A code at bit k of a half word, put into the mantissa of 1024.0 (0x6400), is 1024 + 2^k u; times 2^-k minus
// (1024 / 2^k + 2^(b-1)) is u - 2^(b-1), exactly (one operation on the multiply-add pipe, which has the room; the
// logic pipe is what a decoding step waits for).  bf16 rows stay as they are.
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
__device__ __forceinline__ constexpr uint32_t f16_pair(int v) {          // a small integer (not 0) as an fp16 pair
  const uint32_t m = (uint32_t)(v < 0 ? -v : v);
  int e = 0;
  while ((m >> (e + 1)) != 0) ++e;
  const uint32_t h = (v < 0 ? 0x8000u : 0u) | (uint32_t)(15 + e) << 10 | ((e > 10 ? m >> (e - 10) : m << (10 - e)) & 0x3FFu);
  return h | h << 16;
}
__device__ __forceinline__ constexpr uint32_t f16_inverse(int k) { return (uint32_t)(15 - k) << 10 | (uint32_t)(15 - k) << 26; }   // 2^-k
// Field of BITS bits at bit K of each half of x as fp16 values u - 2^(BITS-1).
template <int BITS, int K>
__device__ __forceinline__ uint32_t field16(uint32_t x) {
  constexpr uint32_t mask = ((1u << BITS) - 1) << K;
  return hfma2(and_or(x, mask | mask << 16, 0x64006400u), f16_inverse(K), f16_pair(-(1024 >> K) - (1 << (BITS - 1))));
}
// The four fields of BITS bits of each half of x.
template <int BITS>
__device__ __forceinline__ void fields16(uint32_t x, uint32_t* o) {
  if constexpr (BITS == 4) {
    o[0] = field16<4, 0>(x);
    o[1] = field16<4, 4>(x);
    o[2] = field16<4, 0>(x >> 8);
    o[3] = field16<4, 4>(x >> 8);
  } else {
    o[0] = field16<3, 0>(x);
    o[1] = field16<3, 3>(x);
    o[2] = field16<3, 6>(x);
    o[3] = field16<3, 6>(x >> 3);
  }
}
template <int BITS>
__device__ __forceinline__ constexpr int pair16_lo(int j) { return BITS >= 8 ? 2 * j : j; }
template <int BITS>
__device__ __forceinline__ constexpr int pair16_hi(int j) { return BITS >= 8 ? 2 * j + 1 : j + 4; }
template <int BITS, int N, int L>
__device__ __forceinline__ void pairs16(const Lane<BITS, N, L>& r, int i, int idx, uint32_t (&o)[4]) {
  if constexpr (BITS == 16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = r.w[4 * i + j];
  } else if constexpr (BITS == 8) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      o[j] = hfma2(__byte_perm(r.w[2 * i + j / 2], 0x64646464u, j & 1 ? 0x4342 : 0x4140), f16_pair(1), f16_pair(-1152));
  } else if constexpr (BITS == 4) {
    fields16<4>(r.w[i], o);
  } else {
    const uint32_t v = r.bits24(i, idx);
    fields16<3>((v & 0xFFFu) | ((v << 4) & 0x0FFF0000u), o);
  }
}
// Unit i of two rows as eight pairs across the rows: o[e] = (row a, row b) at the unit's element e.
template <int BITS, int N, int L>
__device__ __forceinline__ void cross16(const Lane<BITS, N, L>& a, const Lane<BITS, N, L>& b, int i, int idx, uint32_t (&o)[8]) {
  if constexpr (BITS == 16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o[2 * j] = __byte_perm(a.w[4 * i + j], b.w[4 * i + j], 0x5410);
      o[2 * j + 1] = __byte_perm(a.w[4 * i + j], b.w[4 * i + j], 0x7632);
    }
  } else if constexpr (BITS == 8) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      o[e] = hfma2(and_or(__byte_perm(a.w[2 * i + e / 4], b.w[2 * i + e / 4], ((4 + (e & 3)) << 8) | (e & 3)), 0x00FF00FFu, 0x64006400u),
                   f16_pair(1), f16_pair(-1152));
  } else {
    const uint32_t x = BITS == 4 ? a.w[i] : a.bits24(i, idx), y = BITS == 4 ? b.w[i] : b.bits24(i, idx);
    fields16<BITS>(__byte_perm(x, y, 0x5410), o);
    fields16<BITS>(BITS == 4 ? __byte_perm(x, y, 0x7632) : __byte_perm(x >> 12, y >> 12, 0x5410), o + 4);
  }
}
__device__ __forceinline__ uint32_t pack2_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// bf16 rows: bf16 operands; codes: fp16 operands.
template <int BITS>
__device__ __forceinline__ void mma_rows(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (BITS == 16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace frag
}  // namespace hbl
