// Query and key heads divided by their root mean square, times a gain, and rotated, in one pass; and the backward pass.
//
//   o = r R(g x),  r = 1 / sqrt(mean_d x^2 + eps);   R: c x1 - s x2, c x2 + s x1 on the pairs of the first rot_dim elements
//   t = R^T do,  u = g t,  dx = r (u - x r^2 mean_d(x u)),  dg = sum over rows of t x r
//
// R is linear, so r goes last: one product for each element instead of one before the gain.  The statistic is
// summed in fp64 and r rounded once, the products and sums of the rest are rounded one by one in fp32: o is the plain fp32
// evaluation bit for bit (kv_append_kernel quantizes the same values).  The backward pass is fp32 throughout.
//
// A thread owns what rope_kernel's does: 8 elements of the interleaved layout, 8 + 8 partners of the half layout, 8 of the
// part that is not rotated.  The L lanes of a head add up its statistic; HEADS heads of a token (all of q, or all of k)
// share a thread's gains and the table's pairs, and their loads are in flight together.
#include "hbl_kv_cache.cuh"
#include "hbl_piece.cuh"

namespace hbl {
namespace {

constexpr int kThreads = 256, kForwardBlocksPerSm = 3, kBackwardBlocksPerSm = 2;

struct Part {                          // the queries, or the keys
  const void *x, *gain;
  void* out;                           // forward: o; backward: dx
  const void* grad;                    // backward: do
  float* partial;                      // backward: [blocks][head_dim], NULL: gain's gradient is not wanted
  long x_ts, x_hs, o_ts, o_hs, g_ts, g_hs;
  int n_heads, groups, blocks;
  long units;                          // tokens * groups
};
struct NormArgs {
  Part part[2];
  const int32_t* positions;
  const float4* table;                 // NULL: nothing is rotated
  int* status;
  int gain_bf16, n_pos, rot_dim, head_dim, pieces, rotated;
  float eps;
};

// The pairs of a piece: cosines and sines, two to an element.
template <int PAIRS>
__device__ __forceinline__ void load_pairs(const NormArgs& a, int pos, int piece, float2 (&c)[PAIRS / 2], float2 (&s)[PAIRS / 2]) {
  const float4* row = a.table + ((long)pos * (a.rot_dim / 2) + piece * PAIRS) / 2;      // two pairs to a float4
#pragma unroll
  for (int i = 0; i < PAIRS / 2; ++i) {
    const float4 v = __ldg(row + i);
    c[i] = make_float2(v.x, v.z);
    s[i] = make_float2(v.y, v.w);
  }
}

// Where a thread is in its part's units (a token's HEADS heads each), and where it goes next.
struct Walker {
  long unit, units, step;
  int t, group, groups, step_t, step_group;       // the token, and which of its groups of heads
  __device__ __forceinline__ Walker(const Part& w, int block, int slots, int slot) {
    groups = w.groups;
    units = w.units;
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

// Thread blocks stay and walk over the units of their part.  A thread copies its pieces of the next unit to shared memory, where
// only it reads them, while it works on the current one's.
template <typename T, bool INTERLEAVED, int HEADS>
struct ForwardGeo {
  static constexpr int BYTES = 8 * sizeof(T), PIECES = INTERLEAVED ? 1 : 2;      // of a thread and head
  static constexpr int STAGE = HEADS * PIECES * BYTES * kThreads;
};
template <typename T, bool INTERLEAVED, int L, int HEADS>
__global__ void __launch_bounds__(kThreads, kForwardBlocksPerSm) norm_rope_kernel(const __grid_constant__ NormArgs a) {
  using G = ForwardGeo<T, INTERLEAVED, HEADS>;
  constexpr int PAIRS = INTERLEAVED ? 4 : 8, SLOTS = kThreads / L, Q = G::BYTES / 16;
  extern __shared__ uint4 ring[];                              // [stage][head][piece][16 bytes of it][thread]
  grid_dependency_wait();
  const bool second = (int)blockIdx.x >= a.part[0].blocks;
  const Part& w = a.part[second];
  const int block = blockIdx.x - (second ? a.part[0].blocks : 0), piece = threadIdx.x % L;
  const bool there = piece < a.pieces, turned = piece < a.rotated, two = !INTERLEAVED && turned;
  const int half = a.rot_dim / 2, d = turned ? piece * 8 : a.rot_dim + (piece - a.rotated) * 8;
  Walker at(w, block, SLOTS, threadIdx.x / L);
  uint4* const mine = ring + threadIdx.x;
  auto slot = [&](int stage, int i, int half_of) { return mine + (stage * (G::STAGE / 16) + (i * G::PIECES + half_of) * Q * kThreads); };
  auto copy = [&](int stage) {
    if (there && at.live()) {
      const int h0 = at.group * HEADS;
      const T* x = static_cast<const T*>(w.x) + at.t * w.x_ts + h0 * w.x_hs + d;
#pragma unroll
      for (int i = 0; i < HEADS; ++i)
        if (h0 + i < w.n_heads) {
#pragma unroll
          for (int b = 0; b < Q; ++b) {
            copy_async16(slot(stage, i, 0) + b * kThreads, reinterpret_cast<const uint4*>(x + i * w.x_hs) + b);
            if (two) copy_async16(slot(stage, i, 1) + b * kThreads, reinterpret_cast<const uint4*>(x + i * w.x_hs + half) + b);
          }
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto fetch = [&](int stage, int i, int half_of, float2 (&f)[4]) {
    Piece<T> p;
    p.load_from(slot(stage, i, half_of), kThreads);
    p.get(*reinterpret_cast<float(*)[8]>(f));
  };
  auto position = [&]() { return a.table != nullptr && at.live() ? __ldg(a.positions + at.t) : 0; };
  copy(0);
  int pos = position();
  float2 g[4], g2[4];
  if (there) load_gain(w.gain, a.gain_bf16, d, *reinterpret_cast<float(*)[8]>(g));
  if (two) load_gain(w.gain, a.gain_bf16, d + half, *reinterpret_cast<float(*)[8]>(g2));
  const double inv_dim = 1.0 / a.head_dim;
  int stage = 0;
  for (long u0 = (long)block * SLOTS; u0 < w.units; u0 += (long)w.blocks * SLOTS, stage ^= 1) {
    float2 c[PAIRS / 2], s[PAIRS / 2];
    bool good = at.live();
    if (a.table != nullptr) {
      if (pos < 0 || pos >= a.n_pos) {
        report_device_error(a.status, HBL_ERR_RANGE);
        good = false;
      }
      if (turned && good) load_pairs<PAIRS>(a, pos, piece, c, s);
    }
    const int h0 = at.group * HEADS, n = there ? min(HEADS, w.n_heads - h0) : 0;
    T* out = static_cast<T*>(w.out) + at.t * w.o_ts + h0 * w.o_hs + d;
    const bool filled = at.live();
    at.next();
    pos = position();
    copy(stage ^ 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    // the heads' statistics side by side: each is a chain of fp64 operations
    double sum[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      float2 f[4];
      sum[i] = 0.0;
      if (i < n && filled) {
        fetch(stage, i, 0, f);
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[i] = fma((double)f[k].y, (double)f[k].y, fma((double)f[k].x, (double)f[k].x, sum[i]));
        if (two) {
          fetch(stage, i, 1, f);
#pragma unroll
          for (int k = 0; k < 4; ++k) sum[i] = fma((double)f[k].y, (double)f[k].y, fma((double)f[k].x, (double)f[k].x, sum[i]));
        }
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
      if (piece % HEADS == i) of_lane = sum[i];
    const float root = inverse_root(fma(of_lane, inv_dim, (double)a.eps));
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      const float r = __shfl_sync(0xffffffffu, root, i, L);
      if (i >= n || !good) continue;
      float2 f[4];
      fetch(stage, i, 0, f);
      Piece<T> o;
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k] = mul2(f[k], g[k]);
      if (turned) {
        if constexpr (INTERLEAVED) {
          float* y = reinterpret_cast<float*>(f);
          const float *cc = reinterpret_cast<const float*>(c), *ss = reinterpret_cast<const float*>(s);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float x1 = y[2 * k], x2 = y[2 * k + 1];
            y[2 * k] = __fsub_rn(__fmul_rn(x1, cc[k]), __fmul_rn(x2, ss[k]));
            y[2 * k + 1] = __fadd_rn(__fmul_rn(x2, cc[k]), __fmul_rn(x1, ss[k]));
          }
        } else {
          float2 e[4];
          fetch(stage, i, 1, e);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 x1 = f[k], x2 = mul2(e[k], g2[k]);
            f[k] = sub2(mul2(x1, c[k]), mul2(x2, s[k]));
            e[k] = mul2(add2(mul2(x2, c[k]), mul2(x1, s[k])), make_float2(r, r));
          }
          o.set(*reinterpret_cast<float(*)[8]>(e));
          o.store(out + i * w.o_hs + half);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k] = mul2(f[k], make_float2(r, r));
      o.set(*reinterpret_cast<float(*)[8]>(f));
      o.store(out + i * w.o_hs);
    }
  }
}

// The same walk; a thread keeps its piece of the head, so that its share of dg stays in registers.  The block's shares are added
// in shared memory in the order of its threads, the blocks' by gain_grad_kernel.
template <typename T, bool INTERLEAVED, int L, int HEADS>
struct BackwardGeo {
  using F = ForwardGeo<T, INTERLEAVED, HEADS>;
  static constexpr int N = 8 * F::PIECES, PITCH = L * N + 4, SLOTS = kThreads / L;
  static constexpr int RING = 2 * 2 * F::STAGE, SHARES = SLOTS * PITCH * 4, SMEM = RING > SHARES ? RING : SHARES;
};
template <typename T, bool INTERLEAVED, int L, int HEADS>
__global__ void __launch_bounds__(kThreads, kBackwardBlocksPerSm) norm_rope_grad_kernel(const __grid_constant__ NormArgs a) {
  using G = ForwardGeo<T, INTERLEAVED, HEADS>;
  using B = BackwardGeo<T, INTERLEAVED, L, HEADS>;
  constexpr int PAIRS = INTERLEAVED ? 4 : 8, SLOTS = B::SLOTS, N = B::N, Q = G::BYTES / 16, P = G::PIECES;
  extern __shared__ uint4 ring[];                              // [stage][x, do][head][piece][16 bytes of it][thread]
  grid_dependency_wait();
  const bool second = (int)blockIdx.x >= a.part[0].blocks;
  const Part& w = a.part[second];
  const int block = blockIdx.x - (second ? a.part[0].blocks : 0), piece = threadIdx.x % L;
  const bool there = piece < a.pieces, turned = piece < a.rotated, two = !INTERLEAVED && turned;
  const int half = a.rot_dim / 2, d = turned ? piece * 8 : a.rot_dim + (piece - a.rotated) * 8;
  Walker at(w, block, SLOTS, threadIdx.x / L);
  uint4* const mine = ring + threadIdx.x;
  auto slot = [&](int stage, int which, int i, int half_of) {
    return mine + ((stage * 2 + which) * (G::STAGE / 16) + (i * P + half_of) * Q * kThreads);
  };
  auto copy = [&](int stage) {
    if (there && at.live()) {
      const int h0 = at.group * HEADS;
      const T* x = static_cast<const T*>(w.x) + at.t * w.x_ts + h0 * w.x_hs + d;
      const T* y = static_cast<const T*>(w.grad) + at.t * w.g_ts + h0 * w.g_hs + d;
#pragma unroll
      for (int i = 0; i < HEADS; ++i)
        if (h0 + i < w.n_heads) {
#pragma unroll
          for (int b = 0; b < Q; ++b) {
            copy_async16(slot(stage, 0, i, 0) + b * kThreads, reinterpret_cast<const uint4*>(x + i * w.x_hs) + b);
            copy_async16(slot(stage, 1, i, 0) + b * kThreads, reinterpret_cast<const uint4*>(y + i * w.g_hs) + b);
            if (two) {
              copy_async16(slot(stage, 0, i, 1) + b * kThreads, reinterpret_cast<const uint4*>(x + i * w.x_hs + half) + b);
              copy_async16(slot(stage, 1, i, 1) + b * kThreads, reinterpret_cast<const uint4*>(y + i * w.g_hs + half) + b);
            }
          }
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto fetch = [&](const uint4* from, float2* f) {
    Piece<T> p;
    p.load_from(from, kThreads);
    p.get(*reinterpret_cast<float(*)[8]>(f));
  };
  auto position = [&]() { return a.table != nullptr && at.live() ? __ldg(a.positions + at.t) : 0; };
  copy(0);
  int pos = position();
  float2 g[N / 2], acc[N / 2];
#pragma unroll
  for (int k = 0; k < N / 2; ++k) g[k] = acc[k] = make_float2(0.f, 0.f);
  if (there) load_gain(w.gain, a.gain_bf16, d, *reinterpret_cast<float(*)[8]>(g));
  if constexpr (!INTERLEAVED)
    if (two) load_gain(w.gain, a.gain_bf16, d + half, *reinterpret_cast<float(*)[8]>(g + 4));
  const float inv_dim = 1.f / (float)a.head_dim;
  int stage = 0;
  for (long u0 = (long)block * SLOTS; u0 < w.units; u0 += (long)w.blocks * SLOTS, stage ^= 1) {
    float2 c[PAIRS / 2], s[PAIRS / 2];
    bool good = at.live();
    if (a.table != nullptr) {
      if (pos < 0 || pos >= a.n_pos) {
        report_device_error(a.status, HBL_ERR_RANGE);
        good = false;
      }
      if (turned && good) load_pairs<PAIRS>(a, pos, piece, c, s);
    }
    const int h0 = at.group * HEADS, n = there && good ? min(HEADS, w.n_heads - h0) : 0;
    T* out = static_cast<T*>(w.out) + at.t * w.o_ts + h0 * w.o_hs + d;
    at.next();
    pos = position();
    copy(stage ^ 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      float2 f[N / 2], y[N / 2], sums = make_float2(0.f, 0.f), dots = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < N / 2; ++k) f[k] = y[k] = make_float2(0.f, 0.f);
      if (i < n) {
        fetch(slot(stage, 0, i, 0), f);
        fetch(slot(stage, 1, i, 0), y);
        if constexpr (!INTERLEAVED)
          if (two) {
            fetch(slot(stage, 0, i, 1), f + 4);
            fetch(slot(stage, 1, i, 1), y + 4);
          }
        if (turned) {                                          // the transposed rotation
          if constexpr (INTERLEAVED) {
            const float *cc = reinterpret_cast<const float*>(c), *ss = reinterpret_cast<const float*>(s);
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = make_float2(fmaf(y[k].y, ss[k], y[k].x * cc[k]), fmaf(-y[k].x, ss[k], y[k].y * cc[k]));
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
        for (int k = 0; k < N / 2; ++k) {
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
      if (i >= n) continue;
      const float r = 1.f / sqrtf(fmaf(sum, inv_dim, a.eps)), m = -r * (r * r * (dot * inv_dim));
      const float2 rr = make_float2(r, r), mm = make_float2(m, m);
#pragma unroll
      for (int k = 0; k < N / 2; ++k) {
        acc[k] = fma2(y[k], mul2(f[k], rr), acc[k]);
        f[k] = fma2(f[k], mm, mul2(mul2(y[k], g[k]), rr));
      }
      Piece<T> o;
      o.set(*reinterpret_cast<float(*)[8]>(f));
      o.store(out + i * w.o_hs);
      if constexpr (!INTERLEAVED)
        if (two) {
          o.set(*reinterpret_cast<float(*)[8]>(f + 4));
          o.store(out + i * w.o_hs + half);
        }
    }
  }
  if (w.partial == nullptr) return;
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();                                             // nobody reads or fills the ring any more
  float* share = reinterpret_cast<float*>(ring);
#pragma unroll
  for (int k = 0; k < N / 4; ++k)
    *reinterpret_cast<float4*>(share + (threadIdx.x / L) * B::PITCH + piece * N + 4 * k) = make_float4(acc[2 * k].x, acc[2 * k].y, acc[2 * k + 1].x, acc[2 * k + 1].y);
  __syncthreads();
  for (int e = threadIdx.x; e < a.head_dim; e += kThreads) {
    // element e of the head: which thread's, and which of its
    int from;
    if (INTERLEAVED) from = e;
    else if (e < a.rot_dim) from = (e % half) / 8 * N + (e >= half ? 8 : 0) + e % 8;
    else from = (a.rotated + (e - a.rot_dim) / 8) * N + e % 8;
    float sum = 0.f;
#pragma unroll 8
    for (int i = 0; i < SLOTS; ++i) sum += share[i * B::PITCH + from];
    w.partial[(long)block * a.head_dim + e] = sum;
  }
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
  n.table = reinterpret_cast<const float4*>(c.table);
  n.gain_bf16 = c.gain_dtype == HBL_BF16;
  n.n_pos = c.n_pos; n.rot_dim = c.table != nullptr ? c.rot_dim : 0; n.head_dim = c.head_dim; n.eps = c.norm_eps;
  n.rotated = n.rot_dim / (c.interleaved ? 8 : 16);
  n.pieces = n.rotated + (c.head_dim - n.rot_dim) / 8;
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
template <typename T, bool INTERLEAVED, int L, int HEADS>
int launch_forward(NormArgs& n, int tokens, cudaStream_t s) {
  set_units(n, tokens, HEADS);
  deal_blocks(n, kThreads / L, (long)sm_count() * kForwardBlocksPerSm);
  auto kern = norm_rope_kernel<T, INTERLEAVED, L, HEADS>;
  constexpr int bytes = 2 * ForwardGeo<T, INTERLEAVED, HEADS>::STAGE;
  HBL_ALLOW_DYNAMIC_SMEM(kern, bytes);
  HBL_CUDA_OK(launch_waiting(kern, dim3(n.part[0].blocks + n.part[1].blocks), dim3(kThreads), bytes, s, n));
  note_launch();
  return HBL_OK;
}
template <typename T, bool INTERLEAVED, int L, int HEADS>
int launch_backward(NormArgs& n, int tokens, cudaStream_t s) {
  set_units(n, tokens, HEADS);
  deal_blocks(n, kThreads / L, norm_rope_grad_blocks());
  if (n.part[1].partial != nullptr) n.part[1].partial += (long)n.part[0].blocks * n.head_dim;
  auto kern = norm_rope_grad_kernel<T, INTERLEAVED, L, HEADS>;
  constexpr int bytes = BackwardGeo<T, INTERLEAVED, L, HEADS>::SMEM;
  HBL_ALLOW_DYNAMIC_SMEM(kern, bytes);
  HBL_CUDA_OK(launch_waiting(kern, dim3(n.part[0].blocks + n.part[1].blocks), dim3(kThreads), bytes, s, n));
  note_launch();
  return HBL_OK;
}
template <typename T, bool INTERLEAVED, int L>
int launch_lanes(NormArgs& n, int tokens, bool backward, cudaStream_t s) {
  const bool many = (long)tokens * (n.part[0].n_heads + n.part[1].n_heads) * L >= (long)sm_count() * 2048 * 4;
  if (backward) return many ? launch_backward<T, INTERLEAVED, L, sizeof(T) == 2 ? 2 : 1>(n, tokens, s) : launch_backward<T, INTERLEAVED, L, 1>(n, tokens, s);
  return many ? launch_forward<T, INTERLEAVED, L, sizeof(T) == 2 ? 4 : 2>(n, tokens, s) : launch_forward<T, INTERLEAVED, L, 1>(n, tokens, s);
}
template <typename T, bool INTERLEAVED>
int launch_type(NormArgs& n, int tokens, bool backward, cudaStream_t s) {
  if (n.pieces <= 8) return launch_lanes<T, INTERLEAVED, 8>(n, tokens, backward, s);
  if (n.pieces <= 16) return launch_lanes<T, INTERLEAVED, 16>(n, tokens, backward, s);
  return launch_lanes<T, INTERLEAVED, 32>(n, tokens, backward, s);
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
    g.out[i] = c.part[i].grad_gain;
    n.part[i].partial = g.out[i] != nullptr ? partial : nullptr;
    any |= g.out[i] != nullptr;
  }
  const int rc = c.tokens > 0 ? launch_any(n, c, true, s) : HBL_OK;      // (no tokens: no shares, and zeros for their sum)
  if (rc != HBL_OK || !any) return rc;
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
