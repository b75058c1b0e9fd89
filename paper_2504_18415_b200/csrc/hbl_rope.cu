// Rotary positions: o1 = c x1 - s x2, o2 = c x2 + s x1 on the pairs of a head's first rot_dim elements, and the table of
// (c, s) they are rotated by.
//
// The table is made once per model in fp64 (an fp32 angle loses its fraction at far positions); the rotation itself is
// fp32, products and sums rounded one by one, so that it is the plain fp32 evaluation bit for bit: a key that is
// quantized afterwards lands on the same side of every rounding border.
//
// Bound by HBM: every element is read and written once (16384 tokens of 32 heads of 128 in bf16: 46 us, 6.0 TB/s; 3333 of 20
// heads in fp32, half of each rotated: 13.4 us, 5.2 TB/s).  A thread owns one piece of a head (8 elements of the
// interleaved layout, 8 + 8 of the half layout, 8 of the part that is only copied) for up to HEADS heads of a token, so the
// 8 (4) pairs of the table it needs are loaded once for all of them and its HEADS loads are in flight together.
#include "hbl_kv_cache.cuh"
#include "hbl_piece.cuh"

namespace hbl {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxFreq = 128;
struct Freqs { double f[kMaxFreq]; };

__global__ void __launch_bounds__(kThreads)
rope_table_kernel(const __grid_constant__ Freqs freq, int n_freq, double amplitude, int first_pos, long n, float2* __restrict__ table) {
  grid_dependency_wait();
  const long i = (long)blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  const double angle = (double)(first_pos + i / n_freq) * freq.f[i % n_freq];
  double sn, cs;
  sincos(angle, &sn, &cs);
  table[i] = make_float2((float)(amplitude * cs), (float)(amplitude * sn));
}

struct RopeArgs {
  const void* x;
  void* out;
  const int32_t* positions;
  const float4* table;
  int* status;
  long x_ts, x_hs, o_ts, o_hs;
  int tokens, n_heads, n_pos, rot_dim, pieces, rotated, groups, backward;
  long items;
};

template <typename T, bool INTERLEAVED, int HEADS>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ RopeArgs a) {
  grid_dependency_wait();
  const long item = (long)blockIdx.x * kThreads + threadIdx.x;
  if (item >= a.items) return;
  // item = ((token * groups) + head group) * pieces + piece: neighbouring threads take neighbouring pieces
  const int piece = (int)(item % a.pieces);
  const long rest = item / a.pieces;
  const int t = (int)(rest / a.groups), h0 = (int)(rest % a.groups) * HEADS;
  const int pos = __ldg(a.positions + t);
  const int n = min(HEADS, a.n_heads - h0);
  const bool turned = piece < a.rotated;
  // where the piece (and, in the half layout, its partner) lies in the head
  const int half = a.rot_dim / 2;
  const int d = turned ? piece * 8 : a.rot_dim + (piece - a.rotated) * 8;
  const T* x = static_cast<const T*>(a.x) + t * a.x_ts + h0 * a.x_hs + d;
  T* out = static_cast<T*>(a.out) + t * a.o_ts + h0 * a.o_hs + d;
  constexpr bool kTwo = !INTERLEAVED;
  Piece<T> p[HEADS], r[HEADS];
#pragma unroll
  for (int i = 0; i < HEADS; ++i)
    if (i < n) {
      p[i].load(x + i * a.x_hs);
      if (kTwo && turned) r[i].load(x + i * a.x_hs + half);
    }
  if (pos < 0 || pos >= a.n_pos) {
    report_device_error(a.status, HBL_ERR_RANGE);
    return;
  }
  if (!turned) {
    if (a.x == a.out) return;                                  // in place: already there
#pragma unroll
    for (int i = 0; i < HEADS; ++i)
      if (i < n) p[i].store(out + i * a.o_hs);
    return;
  }
  constexpr int PAIRS = INTERLEAVED ? 4 : 8;
  float c[PAIRS], s[PAIRS];
  const float4* row = a.table + ((long)pos * half + piece * PAIRS) / 2;      // two pairs to a float4
#pragma unroll
  for (int i = 0; i < PAIRS / 2; ++i) {
    const float4 v = __ldg(row + i);
    c[2 * i] = v.x; s[2 * i] = v.y; c[2 * i + 1] = v.z; s[2 * i + 1] = v.w;
  }
  if (a.backward) {
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) s[i] = -s[i];
  }
#pragma unroll
  for (int i = 0; i < HEADS; ++i)
    if (i < n) {
      float f[8];
      p[i].get(f);
      if constexpr (INTERLEAVED) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float x1 = f[2 * k], x2 = f[2 * k + 1];
          f[2 * k] = __fsub_rn(__fmul_rn(x1, c[k]), __fmul_rn(x2, s[k]));
          f[2 * k + 1] = __fadd_rn(__fmul_rn(x2, c[k]), __fmul_rn(x1, s[k]));
        }
        p[i].set(f);
        p[i].store(out + i * a.o_hs);
      } else {
        float g[8];
        r[i].get(g);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float x1 = f[k], x2 = g[k];
          f[k] = __fsub_rn(__fmul_rn(x1, c[k]), __fmul_rn(x2, s[k]));
          g[k] = __fadd_rn(__fmul_rn(x2, c[k]), __fmul_rn(x1, s[k]));
        }
        p[i].set(f);
        r[i].set(g);
        p[i].store(out + i * a.o_hs);
        r[i].store(out + i * a.o_hs + half);
      }
    }
}

template <typename T, bool INTERLEAVED, int HEADS>
int launch_one(RopeArgs& a, cudaStream_t s) {
  a.groups = (a.n_heads + HEADS - 1) / HEADS;
  a.items = (long)a.tokens * a.groups * a.pieces;
  const long blocks = (a.items + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffffL) return HBL_ERR_TOO_LARGE;
  HBL_CUDA_OK(launch_waiting(rope_kernel<T, INTERLEAVED, HEADS>, dim3((unsigned)blocks), dim3(kThreads), 0, s, a));
  note_launch();
  return HBL_OK;
}
// Four heads to a thread once that still leaves every SM a full set of threads; one while the call is small and
// its latency is what counts.
template <typename T, bool INTERLEAVED>
int launch_type(RopeArgs& a, cudaStream_t s) {
  const long one = (long)a.tokens * a.n_heads * a.pieces;
  if (one >= (long)sm_count() * 2048 * 4) return launch_one<T, INTERLEAVED, 4>(a, s);
  return launch_one<T, INTERLEAVED, 1>(a, s);
}

}  // namespace

int launch_rope_table(const double* freq, int n_freq, double amplitude, int first_pos, int n_pos, float* table, cudaStream_t s) {
  Freqs f;
  for (int i = 0; i < n_freq; ++i) f.f[i] = freq[i];
  const long n = (long)n_pos * n_freq;
  if (n == 0) return HBL_OK;
  const long blocks = (n + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffffL) return HBL_ERR_TOO_LARGE;
  HBL_CUDA_OK(launch_waiting(rope_table_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, s, f, n_freq, amplitude, first_pos, n,
                               reinterpret_cast<float2*>(table)));
  note_launch();
  return HBL_OK;
}

int launch_rope(const void* x, int dtype, int tokens, int n_heads, int head_dim, long x_ts, long x_hs, const int32_t* positions,
                const float* table, int n_pos, int rot_dim, int layout, int backward, void* out, long o_ts, long o_hs,
                cudaStream_t s) {
  RopeArgs a{};
  a.x = x; a.out = out; a.positions = positions; a.table = reinterpret_cast<const float4*>(table);
  a.status = device_status_word();
  if (a.status == nullptr) return HBL_ERR_CUDA;
  a.x_ts = x_ts; a.x_hs = x_hs; a.o_ts = o_ts; a.o_hs = o_hs;
  a.tokens = tokens; a.n_heads = n_heads; a.n_pos = n_pos; a.rot_dim = rot_dim; a.backward = backward;
  const bool inter = layout == HBL_ROPE_INTERLEAVED;
  a.rotated = inter ? rot_dim / 8 : rot_dim / 16;
  a.pieces = a.rotated + (head_dim - rot_dim) / 8;
  if (dtype == HBL_BF16) return inter ? launch_type<__nv_bfloat16, true>(a, s) : launch_type<__nv_bfloat16, false>(a, s);
  return inter ? launch_type<float, true>(a, s) : launch_type<float, false>(a, s);
}

}  // namespace hbl
