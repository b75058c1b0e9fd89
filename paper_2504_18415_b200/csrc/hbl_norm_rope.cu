// Query and key heads divided by their root mean square, times a gain, and rotated, in one pass; and the backward pass.
//
//   o = r R(g x),  r = 1 / sqrt(mean_d x^2 + eps);   R: c x1 - s x2, c x2 + s x1 on the pairs of the first rot_dim elements
//   t = R^T do,  u = g t,  dx = r (u - x r^2 mean_d(x u)),  dg = sum over rows of t x r
//
// R is linear, so r goes last: one product for each element instead of one before the gain.  The statistic is
// summed in fp64 and r rounded once, the products and sums of the rest are rounded one by one in fp32: o is the plain fp32
// evaluation bit for bit (kv_append_kernel quantizes the same values).  The backward pass is fp32, but for heads whose mean square and eps
// lie outside 2^-60 .. 2^60: their squares, or r^2, could leave its range, so the statistic is summed in fp64 there, and x r goes
// into the other sum, whose terms are then of u's size.
//
// A thread owns 16 elements of a head; the L lanes of a head add up its statistic.  Thread blocks stay and walk over the call's
// heads, HEADS of a token at a time: the gains are loaded once, the table's pairs once for HEADS heads, and the next ones are
// copied to shared memory while a thread works on the current ones.
//
// Bound by HBM and by what hides its latency: 16384 tokens of 32 and 8 heads of 128 in bf16 62.8 us forward (0.84 of what the bytes
// need), 94.2 us backward (0.83); 8192 in fp32 61.2 and 81.4 (0.85, 0.95).  Registers leave two blocks to an SM (three, spilling: 70 us
// forward, 164 backward); issue slots 60 %.  The loads straight into registers: 73 and 127.  The statistic in fp32 would save 6 us.
#include "hbl_kv_cache.cuh"
#include "hbl_piece.cuh"

namespace hbl {
namespace {

constexpr int kThreads = 256, kForwardBlocksPerSm = 2, kBackwardBlocksPerSm = 2;

struct Part {                          // the queries, or the keys
  const void *x, *gain;
  void* out;                           // forward: o; backward: dx
  const void* grad;                    // backward: do
  float *partial, *grad_gain;          // backward: [blocks][head_dim], NULL: gain's gradient is not wanted
  long x_ts, x_hs, o_ts, o_hs, g_ts, g_hs;
  int n_heads, groups, blocks;
  long units;                          // tokens * groups
};
struct NormArgs {
  Part part[2];
  const int32_t* positions;
  const float2* table;                 // NULL: nothing is rotated
  int* status;
  int gain_bf16, n_pos, rot_dim, head_dim, pieces, rotated, joined;
  float eps;
};

// A thread's 16 elements of a head, 16 bytes at a time: chunk k of lane j of the L' lanes that share a part is the part's chunk
// k L' + j, so that neighbouring lanes read neighbouring bytes.  The partners of the half layout are then a thread's own (chunk k
// and k + N / 2), like those of the interleaved one, which lie in a chunk.  FULL: head_dim is a multiple of 16, so that every
// thread that has chunks at all has N.
template <typename T, bool FULL>
struct Chunks {
  static constexpr int E = 16 / sizeof(T), N = 16 / E;          // elements of a chunk, chunks of a thread
  bool there, turned;                  // any at all; in the rotated part
  int d, step, n;                      // the first one's element, from one to the next, how many
  int pair, pair_step;                 // the first one's pair in the table's row, from one to the next
  __device__ __forceinline__ Chunks(const NormArgs& a, bool interleaved, int lane) {
    turned = lane < a.rotated;
    const int first = turned ? 0 : a.rot_dim, lanes = turned ? a.rotated : a.pieces - a.rotated, j = turned ? lane : lane - a.rotated;
    there = lane < a.pieces;
    d = first + j * E;
    step = lanes * E;
    n = turned ? N : there ? min(N, (a.head_dim - d + step - 1) / step) : 0;
    if (FULL) n = N;
    pair = interleaved ? d / 2 : d;
    pair_step = interleaved ? step / 2 : step;
  }
};
template <typename T>
__device__ __forceinline__ void widen(const uint4& w, float2* f) {     // a chunk
  if constexpr (sizeof(T) == 2) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xFFFF0000u));
  } else {
    f[0] = make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
    f[1] = make_float2(__uint_as_float(w.z), __uint_as_float(w.w));
  }
}
template <typename T>
__device__ __forceinline__ uint4 narrow(const float2* f) {
  if constexpr (sizeof(T) == 2) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[i].x, f[i].y);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  } else {
    return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
  }
}
// The gains of a thread's elements; NULL: ones.
template <typename T, bool FULL>
__device__ __forceinline__ void load_gains(const NormArgs& a, const void* gain, const Chunks<T, FULL>& own, float2 (&g)[8]) {
  constexpr int E = Chunks<T, FULL>::E;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int k = 2 * i / E, d = own.d + k * own.step + 2 * i % E;
    g[i] = make_float2(1.f, 1.f);
    if (gain != nullptr && own.there && k < own.n) {
      if (a.gain_bf16) {
        const uint32_t u = __ldg(static_cast<const uint32_t*>(gain) + d / 2);
        g[i] = make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
      } else {
        g[i] = __ldg(reinterpret_cast<const float2*>(static_cast<const float*>(gain) + d));
      }
    }
  }
}
// The 8 pairs of a thread's elements: cosines and sines, two to an element.
template <bool INTERLEAVED, typename T, bool FULL>
__device__ __forceinline__ void load_pairs(const NormArgs& a, int pos, const Chunks<T, FULL>& own, float2 (&c)[4], float2 (&s)[4]) {
  constexpr int E = Chunks<T, FULL>::E / (INTERLEAVED ? 2 : 1);       // pairs of a chunk
  const float2* row = a.table + (long)pos * (a.rot_dim / 2) + own.pair;
#pragma unroll
  for (int i = 0; i < 4; ++i) {                                // two pairs to a float4
    const float4 v = __ldg(reinterpret_cast<const float4*>(row + (2 * i / E) * own.pair_step + 2 * i % E));
    c[i] = make_float2(v.x, v.z);
    s[i] = make_float2(v.y, v.w);
  }
}

// Where a thread is in its part's units (a token's HEADS heads each).
struct Walker {
  long unit, units, step;
  int t, group, groups, step_t, step_group;       // the token, and which of its groups of heads
  __device__ __forceinline__ Walker(const Part& w, int block, int slots, int slot, bool there) {
    groups = w.groups;
    units = there ? w.units : 0;
    step = (long)w.blocks * slots;
    step_t = (int)(step / groups);
    step_group = (int)(step % groups);
    unit = (long)block * slots + slot;
    t = (int)(unit / groups);
    group = (int)(unit % groups);
  }
  __device__ __forceinline__ void next() {
    unit += step;
    t += step_t;
    group += step_group;
    if (group >= groups) {
      group -= groups;
      ++t;
    }
  }
  __device__ __forceinline__ bool live() const { return unit < units; }
};
// One unit of one tensor to shared memory, [head][chunk][thread], where only the thread itself reads it.
template <int HEADS, typename T, bool FULL>
__device__ __forceinline__ void copy_unit(uint4* to, const void* from, long ts, long hs, const Walker& at, int n_heads, const Chunks<T, FULL>& own) {
  constexpr int N = Chunks<T, FULL>::N;
  if (!at.live()) return;
  const int h0 = at.group * HEADS;
  const T* x = static_cast<const T*>(from) + at.t * ts + h0 * hs + own.d;
#pragma unroll
  for (int i = 0; i < HEADS; ++i)
    if (h0 + i < n_heads) {
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (FULL || k < own.n) copy_async16(to + (i * N + k) * kThreads, reinterpret_cast<const uint4*>(x + i * hs + k * own.step));
    }
}
template <typename T, int HEADS>
constexpr int kUnitWords = HEADS * (int)sizeof(T) * kThreads;    // of 16 bytes, of all threads
// A head's elements out of there; zeros where there are none.
template <typename T, bool FULL>
__device__ __forceinline__ void fetch(const uint4* from, const Chunks<T, FULL>& own, float2 (&f)[8]) {
  constexpr int N = Chunks<T, FULL>::N, P = 8 / N;
#pragma unroll
  for (int k = 0; k < N; ++k)
    widen<T>(FULL || k < own.n ? from[k * kThreads] : make_uint4(0, 0, 0, 0), f + k * P);
}
template <typename T, bool FULL>
__device__ __forceinline__ void store(T* out, const Chunks<T, FULL>& own, const float2 (&f)[8]) {
  constexpr int N = Chunks<T, FULL>::N, P = 8 / N;
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (FULL || k < own.n) *reinterpret_cast<uint4*>(out + k * own.step) = narrow<T>(f + k * P);
}
__device__ __forceinline__ float of(const float2 (&c)[4], int k) { return k & 1 ? c[k / 2].y : c[k / 2].x; }
// A token's position; false (and reported): it has none.
__device__ __forceinline__ bool sound(const NormArgs& a, int pos) {
  if (pos >= 0 && pos < a.n_pos) return true;
  report_device_error(a.status, HBL_ERR_RANGE);
  return false;
}

template <typename T, bool INTERLEAVED, bool FULL, int L, int HEADS>
__global__ void __launch_bounds__(kThreads, kForwardBlocksPerSm) norm_rope_kernel(const __grid_constant__ NormArgs a) {
  constexpr int SLOTS = kThreads / L, WORDS = kUnitWords<T, HEADS>, N = Chunks<T, FULL>::N;
  extern __shared__ uint4 ring[];                              // two units
  grid_dependency_wait();
  const bool second = (int)blockIdx.x >= a.part[0].blocks;
  const Part& w = a.part[second];
  const int block = blockIdx.x - (second ? a.part[0].blocks : 0), lane = threadIdx.x % L;
  const Chunks<T, FULL> own(a, INTERLEAVED, lane);
  Walker at(w, block, SLOTS, threadIdx.x / L, own.there);
  auto copy = [&](int stage) {
    copy_unit<HEADS>(ring + threadIdx.x + stage * WORDS, w.x, w.x_ts, w.x_hs, at, w.n_heads, own);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto position = [&]() { return a.table != nullptr && at.live() ? __ldg(a.positions + at.t) : 0; };
  copy(0);
  int pos = position();
  float2 g[8];
  load_gains(a, w.gain, own, g);
  const double inv_dim = 1.0 / a.head_dim;
  int stage = 0;
  for (long u0 = (long)block * SLOTS; u0 < w.units; u0 += (long)w.blocks * SLOTS, stage ^= 1) {
    float2 c[4], s[4];
    bool good = at.live();
    if (a.table != nullptr) {
      good = sound(a, pos) && good;
      if (own.turned && good) load_pairs<INTERLEAVED>(a, pos, own, c, s);
    }
    const int h0 = at.group * HEADS, n = at.live() ? min(HEADS, w.n_heads - h0) : 0;
    T* out = static_cast<T*>(w.out) + at.t * w.o_ts + h0 * w.o_hs + own.d;
    const uint4* here = ring + threadIdx.x + stage * WORDS;
    at.next();
    pos = position();
    copy(stage ^ 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    // the heads' statistics side by side: each is a chain of fp64 operations
    double sum[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      sum[i] = 0.0;
      if (i < n) {
        float2 f[8];
        fetch(here + i * N * kThreads, own, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[i] = fma((double)f[k].y, (double)f[k].y, fma((double)f[k].x, (double)f[k].x, sum[i]));
      }
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) {
#pragma unroll
      for (int i = 0; i < HEADS; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
    }
    // and one root to a lane
    double of_lane = sum[0];
#pragma unroll
    for (int i = 1; i < HEADS; ++i)
      if (lane % HEADS == i) of_lane = sum[i];
    const float root = inverse_root(fma(of_lane, inv_dim, (double)a.eps));
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      const float r = __shfl_sync(0xffffffffu, root, i, L);
      if (i >= n || !good) continue;
      float2 f[8];
      fetch(here + i * N * kThreads, own, f);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = mul2(f[k], g[k]);
      if (own.turned) {
        if constexpr (INTERLEAVED) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float2 x = mul2(f[k], make_float2(of(c, k), of(c, k))), y = mul2(f[k], make_float2(of(s, k), of(s, k)));
            f[k] = make_float2(__fsub_rn(x.x, y.y), __fadd_rn(x.y, y.x));
          }
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 x1 = f[k], x2 = f[k + 4];
            f[k] = sub2(mul2(x1, c[k]), mul2(x2, s[k]));
            f[k + 4] = add2(mul2(x2, c[k]), mul2(x1, s[k]));
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = mul2(f[k], make_float2(r, r));
      store(out + i * w.o_hs, own, f);
    }
  }
}

// Not the aligned form: the loops before it part a warp's lanes at widths that are no multiple of 32.
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ float of_block(const float* mine, int rank) {       // the same place in another block of the cluster
  uint32_t at;
  float x;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
  return x;
}

// The same walk.  A thread keeps its elements of the head, so that its share of dg stays in registers; the block's shares are added
// in shared memory in the order of its threads, the blocks' by gain_grad_kernel, or, in a small call (`joined`), by the first of them:
// the blocks of a part are then one cluster.
constexpr int kJoined = 8;
template <int L>
struct Shares { static constexpr int PITCH = L * 16 + 4, BYTES = kThreads / L * PITCH * 4; };
template <typename T, bool INTERLEAVED, bool FULL, int L, int HEADS>
__global__ void __launch_bounds__(kThreads, kBackwardBlocksPerSm) norm_rope_grad_kernel(const __grid_constant__ NormArgs a) {
  constexpr int SLOTS = kThreads / L, WORDS = kUnitWords<T, HEADS>, N = Chunks<T, FULL>::N, PITCH = Shares<L>::PITCH;
  extern __shared__ uint4 ring[];                              // two units of x and do; at the end the shares
  grid_dependency_wait();
  const bool second = (int)blockIdx.x >= a.part[0].blocks;
  const Part& w = a.part[second];
  const int block = blockIdx.x - (second ? a.part[0].blocks : 0), lane = threadIdx.x % L;
  const Chunks<T, FULL> own(a, INTERLEAVED, lane);
  Walker at(w, block, SLOTS, threadIdx.x / L, own.there);
  auto copy = [&](int stage) {
    copy_unit<HEADS>(ring + threadIdx.x + 2 * stage * WORDS, w.x, w.x_ts, w.x_hs, at, w.n_heads, own);
    copy_unit<HEADS>(ring + threadIdx.x + (2 * stage + 1) * WORDS, w.grad, w.g_ts, w.g_hs, at, w.n_heads, own);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto position = [&]() { return a.table != nullptr && at.live() ? __ldg(a.positions + at.t) : 0; };
  copy(0);
  int pos = position();
  float2 g[8], acc[8];
  load_gains(a, w.gain, own, g);
#pragma unroll
  for (int k = 0; k < 8; ++k) acc[k] = make_float2(0.f, 0.f);
  const float inv_dim = 1.f / (float)a.head_dim;
  int stage = 0;
  for (long u0 = (long)block * SLOTS; u0 < w.units; u0 += (long)w.blocks * SLOTS, stage ^= 1) {
    float2 c[4], s[4];
    bool good = at.live();
    if (a.table != nullptr) {
      good = sound(a, pos) && good;
      if (own.turned && good) load_pairs<INTERLEAVED>(a, pos, own, c, s);
    }
    const int h0 = at.group * HEADS, n = good ? min(HEADS, w.n_heads - h0) : 0;
    T* out = static_cast<T*>(w.out) + at.t * w.o_ts + h0 * w.o_hs + own.d;
    const uint4* here = ring + threadIdx.x + 2 * stage * WORDS;
    at.next();
    pos = position();
    copy(stage ^ 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      float2 f[8], y[8], sums = make_float2(0.f, 0.f), dots = make_float2(0.f, 0.f);
      if (i < n) {
        fetch(here + i * N * kThreads, own, f);
        fetch(here + WORDS + i * N * kThreads, own, y);
        if (own.turned) {                                      // the transposed rotation
          if constexpr (INTERLEAVED) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float2 z = mul2(y[k], make_float2(of(c, k), of(c, k)));
              y[k] = make_float2(fmaf(y[k].y, of(s, k), z.x), fmaf(-y[k].x, of(s, k), z.y));
            }
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float2 y1 = y[k], z = mul2(y[k + 4], c[k]);
              y[k] = fma2(y[k + 4], s[k], mul2(y1, c[k]));
              y[k + 4] = make_float2(fmaf(-y1.x, s[k].x, z.x), fmaf(-y1.y, s[k].y, z.y));
            }
          }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          sums = fma2(f[k], f[k], sums);
          dots = fma2(f[k], mul2(y[k], g[k]), dots);
        }
      }
      float sum = sums.x + sums.y, dot = dots.x + dots.y;
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
      }
      const float square = fmaf(sum, inv_dim, a.eps);
      const bool within = square > 0x1p-60f && square < 0x1p60f;
      float r = 1.f / sqrtf(square);
      dot *= r;                                                // sum of x r u
      if (__any_sync(0xffffffffu, i < n && !within)) {         // heads whose squares, or r^2, are not for fp32
        double wide = 0.0;
        if (i < n) {
#pragma unroll
          for (int k = 0; k < 8; ++k) wide = fma((double)f[k].y, (double)f[k].y, fma((double)f[k].x, (double)f[k].x, wide));
        }
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) wide += __shfl_xor_sync(0xffffffffu, wide, o);
        const float root = inverse_root(fma(wide, 1.0 / a.head_dim, (double)a.eps));
        float2 own_dots = make_float2(0.f, 0.f);
        if (i < n) {
#pragma unroll
          for (int k = 0; k < 8; ++k) own_dots = fma2(mul2(f[k], make_float2(root, root)), mul2(y[k], g[k]), own_dots);
        }
        float own_dot = own_dots.x + own_dots.y;
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) own_dot += __shfl_xor_sync(0xffffffffu, own_dot, o);
        if (!within) {
          r = root;
          dot = own_dot;
        }
      }
      if (i >= n) continue;
      const float m = -r * (dot * inv_dim);
      const float2 rr = make_float2(r, r), mm = make_float2(m, m);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float2 z = mul2(f[k], rr);
        acc[k] = fma2(y[k], z, acc[k]);
        f[k] = fma2(z, mm, mul2(mul2(y[k], g[k]), rr));
      }
      store(out + i * w.o_hs, own, f);
    }
  }
  if (w.partial == nullptr) return;                            // (all blocks of a part)
  __shared__ float sums[256];
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();                                             // nobody reads or fills the ring any more
  float* share = reinterpret_cast<float*>(ring);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int k = 2 * i / Chunks<T, FULL>::E, d = own.d + k * own.step + 2 * i % Chunks<T, FULL>::E;
    if (own.there && k < own.n) *reinterpret_cast<float2*>(share + (threadIdx.x / L) * PITCH + d) = acc[i];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.head_dim; e += kThreads) {
    float sum = 0.f;
#pragma unroll 8
    for (int i = 0; i < SLOTS; ++i) sum += share[i * PITCH + e];
    if (a.joined) sums[e] = sum;
    else w.partial[(long)block * a.head_dim + e] = sum;
  }
  if (!a.joined) return;
  cluster_sync();
  if (block == 0)
    for (int e = threadIdx.x; e < a.head_dim; e += kThreads) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kJoined; ++i) sum += of_block(&sums[e], i);
      w.grad_gain[e] = sum;
    }
  cluster_sync();                                              // nobody leaves before it has been read
}

// dg = the blocks' shares added up, 32 elements to a block: 32 warps take a row of shares each in turn, then their sums
// in the warps' order.
struct GainArgs {
  const float* partial[2];
  float* out[2];
  int blocks[2], head_dim;
};
__global__ void __launch_bounds__(1024) gain_grad_kernel(const __grid_constant__ GainArgs a) {
  __shared__ float share[32][33];
  grid_dependency_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane, which = blockIdx.y;
  if (a.out[which] == nullptr) return;
  float sum = 0.f;
  if (e < a.head_dim)
    for (int b = warp; b < a.blocks[which]; b += 32) sum += a.partial[which][(long)b * a.head_dim + e];
  share[warp][lane] = sum;
  __syncthreads();
  if (warp != 0 || e >= a.head_dim) return;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) sum += share[i][lane];
  a.out[which][e] = sum;
}

void set_pieces(NormArgs& n, const NormRopeCall& c) {
  n.positions = c.positions;
  n.table = reinterpret_cast<const float2*>(c.table);
  n.gain_bf16 = c.gain_dtype == HBL_BF16;
  n.n_pos = c.n_pos; n.rot_dim = c.table != nullptr ? c.rot_dim : 0; n.head_dim = c.head_dim; n.eps = c.norm_eps;
  n.rotated = n.rot_dim / 16;
  n.pieces = (c.head_dim + 15) / 16;
  for (int i = 0; i < 2; ++i) {
    const NormRopePart& s = c.part[i];
    Part& d = n.part[i];
    d.x = s.x; d.gain = s.gain; d.out = s.out; d.grad = s.grad;
    d.x_ts = s.x_ts; d.x_hs = s.x_hs; d.o_ts = s.o_ts; d.o_hs = s.o_hs; d.g_ts = s.g_ts; d.g_hs = s.g_hs;
    d.n_heads = s.n_heads;
  }
}
void set_units(NormArgs& n, int tokens, int heads) {
  for (Part& d : n.part) {
    d.groups = (d.n_heads + heads - 1) / heads;
    d.units = (long)tokens * d.groups;
  }
}

// Blocks for the two parts by their units, at most `most` (and one more, where a part would get none).
void deal_blocks(NormArgs& n, int slots, long most) {
  for (Part& d : n.part) {
    const long share = most * d.units / (n.part[0].units + n.part[1].units), need = (d.units + slots - 1) / slots;
    d.blocks = (int)(need < share ? need : share < 1 && need > 0 ? 1 : share);
  }
}
template <typename T, bool INTERLEAVED, bool FULL, int L, int HEADS>
int launch_forward(NormArgs& n, int tokens, cudaStream_t s) {
  set_units(n, tokens, HEADS);
  deal_blocks(n, kThreads / L, (long)sm_count() * kForwardBlocksPerSm);
  auto kern = norm_rope_kernel<T, INTERLEAVED, FULL, L, HEADS>;
  constexpr int bytes = 2 * 16 * kUnitWords<T, HEADS>;
  HBL_ALLOW_DYNAMIC_SMEM(kern, bytes);
  HBL_CUDA_OK(launch_waiting(kern, dim3(n.part[0].blocks + n.part[1].blocks), dim3(kThreads), bytes, s, n));
  note_launch();
  return HBL_OK;
}
template <typename T, bool INTERLEAVED, bool FULL, int L, int HEADS>
int launch_backward(NormArgs& n, int tokens, cudaStream_t s) {
  set_units(n, tokens, HEADS);
  deal_blocks(n, kThreads / L, norm_rope_grad_blocks());
  // One launch instead of two while a part's units are at most four to a place of its cluster (16 tokens of 32 and 8 heads: 18.3 us
  // with two, 16.4 with one, which the host takes).
  const long places = kJoined * (kThreads / L);
  n.joined = (n.part[0].partial != nullptr || n.part[1].partial != nullptr) && n.part[0].units <= 4 * places && n.part[1].units <= 4 * places;
  if (n.joined)
    for (Part& d : n.part) d.blocks = d.units > 0 ? kJoined : 0;
  if (n.part[1].partial != nullptr) n.part[1].partial += (long)n.part[0].blocks * n.head_dim;
  auto kern = norm_rope_grad_kernel<T, INTERLEAVED, FULL, L, HEADS>;
  constexpr int units = 4 * 16 * kUnitWords<T, HEADS>, bytes = units > Shares<L>::BYTES ? units : Shares<L>::BYTES;
  HBL_ALLOW_DYNAMIC_SMEM(kern, bytes);
  HBL_CUDA_OK(launch_waiting_clusters(kern, dim3(n.part[0].blocks + n.part[1].blocks), dim3(kThreads), bytes, s, n.joined ? kJoined : 1, n));
  note_launch();
  return HBL_OK;
}
// Several heads to a unit once there are as many units as places for them (1024 tokens of 32 and 8 heads: 8.8 us; one to a unit
// 9.5), one while the call is small (and for a head_dim that is no multiple of 16).
template <typename T, bool INTERLEAVED, int L>
int launch_lanes(NormArgs& n, int tokens, bool backward, cudaStream_t s) {
  constexpr int F = sizeof(T) == 2 ? 4 : 2;
  const long places = (long)sm_count() * kForwardBlocksPerSm * (kThreads / L), heads = (long)tokens * (n.part[0].n_heads + n.part[1].n_heads);
  const bool full = n.head_dim % 16 == 0, many = full && heads >= places * F;
  if (backward) {
    if (many) return launch_backward<T, INTERLEAVED, true, L, F / 2>(n, tokens, s);
    return full ? launch_backward<T, INTERLEAVED, true, L, 1>(n, tokens, s) : launch_backward<T, INTERLEAVED, false, L, 1>(n, tokens, s);
  }
  if (many) return launch_forward<T, INTERLEAVED, true, L, F>(n, tokens, s);
  return full ? launch_forward<T, INTERLEAVED, true, L, 1>(n, tokens, s) : launch_forward<T, INTERLEAVED, false, L, 1>(n, tokens, s);
}
template <typename T, bool INTERLEAVED>
int launch_type(NormArgs& n, int tokens, bool backward, cudaStream_t s) {
  if (n.pieces <= 4) return launch_lanes<T, INTERLEAVED, 4>(n, tokens, backward, s);
  if (n.pieces <= 8) return launch_lanes<T, INTERLEAVED, 8>(n, tokens, backward, s);
  return launch_lanes<T, INTERLEAVED, 16>(n, tokens, backward, s);
}
int launch_any(NormArgs& n, const NormRopeCall& c, bool backward, cudaStream_t s) {
  n.status = device_status_word();
  if (n.status == nullptr) return HBL_ERR_CUDA;
  if (c.dtype == HBL_BF16)
    return c.interleaved ? launch_type<__nv_bfloat16, true>(n, c.tokens, backward, s) : launch_type<__nv_bfloat16, false>(n, c.tokens, backward, s);
  return c.interleaved ? launch_type<float, true>(n, c.tokens, backward, s) : launch_type<float, false>(n, c.tokens, backward, s);
}

}  // namespace

// Thread blocks of the backward kernel at most (and one more, where a part would get none).
int norm_rope_grad_blocks() { return sm_count() * kBackwardBlocksPerSm; }

int launch_norm_rope(const NormRopeCall& c, cudaStream_t s) {
  NormArgs n{};
  set_pieces(n, c);
  return launch_any(n, c, false, s);
}

int launch_norm_rope_grad(const NormRopeCall& c, float* partial, cudaStream_t s) {
  NormArgs n{};
  set_pieces(n, c);
  GainArgs g{};
  bool any = false;
  for (int i = 0; i < 2; ++i) {
    g.out[i] = n.part[i].grad_gain = c.part[i].grad_gain;
    n.part[i].partial = g.out[i] != nullptr ? partial : nullptr;
    any |= g.out[i] != nullptr;
  }
  const int rc = c.tokens > 0 ? launch_any(n, c, true, s) : HBL_OK;      // (no tokens: no shares, and zeros for their sum)
  if (rc != HBL_OK || !any || n.joined) return rc;
  for (int i = 0; i < 2; ++i) {
    g.partial[i] = n.part[i].partial;
    g.blocks[i] = n.part[i].blocks;
  }
  g.head_dim = c.head_dim;
  HBL_CUDA_OK(launch_waiting(gain_grad_kernel, dim3((c.head_dim + 31) / 32, 2), dim3(1024), 0, s, g));
  note_launch();
  return HBL_OK;
}

}  // namespace hbl
