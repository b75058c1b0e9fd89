// Attention of many query rows over the paged cache on the 5th-generation tensor cores: prompts and chunks of them.
//
//   S = Q ck^T (tcgen05.mma, fp32 in tensor memory);  s = sm_scale ks_j S;  p = 2^(s - m);  O += (p vs_j) cv
//
// Q and ck are bf16 operands (codes are exact).  bf16 rows: p is rounded to bf16, as cv is.  Codes: p vs_j goes to fp16
// against a running power of two above the value scales (eight times finer), cv is exact in fp16, too.
//
// A work item is 128 * NSUB query rows of one key head (row r: token r / group, head r % group, so that the heads that
// share a key head share its tiles) against one piece of the keys.  One thread block per SM, which goes on to the items of
// blocks that have not started:
//   warps 0-3, 4-7   softmax of sub-tile 0, 1: scores out of tensor memory, maximum, exponentials,
//                    P back into tensor memory as bf16 in the place of the scores; at the end O out of tensor memory
//   warps 8-11       producers: the tiles of keys and values into shared memory, 128-byte swizzle.  Codes become bf16
//                    (exactly) on the way; values beyond the sequence become zeros, whatever the cache holds there
//   warp 12          issues the matrix instructions;  warps 13, 14: the queries into shared memory;  warp 15: looks up the items
// The two sub-tiles alternate on the tensor core: while one's scores are being exponentiated the other's products run.
// Bound by the tensor core and the exponential unit alike at head_dim 128 (256 x 128 scores: 2048 cycles each); a tile takes
// some 3300 (8192-token prompt of 32 heads 490 us, 1120 TFLOP/s while the clock holds; 4096 of 16 heads 72 us, 950).  Over
// codes some 5500, because the widening takes the producers as long (512 queries over 16384 tokens at 8 bits 220 us).
//
// The order of the elements inside each group of 8 of a head is free for Q K^T as long as Q and K agree, and for V it only
// names the columns of O: codes are widened in the order that takes least work (hbl_attn_frag.cuh, `pairs`), the
// queries are put into the same order when they are loaded, and O's columns are put back when they are written.
//
// The maximum is only raised when a score exceeds it by more than 2^8; only then is O rescaled, by the softmax
// threads themselves (the scores' barrier says that the products before it are complete, so O is at rest).
#include "hbl_attn_frag.cuh"
#include "hbl_pipeline.cuh"

namespace hbl {
namespace {

using namespace frag;
using namespace pipe;

constexpr int kThreads = 512;
constexpr float kLazy = 8.f;
constexpr uint32_t kTmemCols = 512;
// The next item is asked for this many tiles before the end of the one at work (2 .. 6 within 3 %).  Asked for at its
// beginning: 4096-token prompt of 16 heads 96 us (72), 2048 of 32 heads 61 (50), four of those 206 (184).
constexpr int kNearEnd = 4;

template <int D>
struct TileGeo {
  static constexpr int NSUB = D == 256 ? 1 : 2;                // sub-tiles of 128 rows
  static constexpr int BK = D == 256 ? 64 : 128;               // keys per tile
  static constexpr int ROWS = 128 * NSUB;
  static constexpr int STAGES = D == 64 ? 3 : 2;
  static constexpr int Q_BYTES = 128 * D * 2, KV_BYTES = BK * D * 2;
  static constexpr int HALF = BK * 128;                        // 64 elements wide column of a key / value tile
  static constexpr int OUT_PITCH = 80, OUT_BYTES = 32 * OUT_PITCH;   // a warp's 32 rows of 64 bytes on their way out
  static constexpr size_t SMEM = (size_t)NSUB * Q_BYTES + (size_t)STAGES * 2 * KV_BYTES + (size_t)STAGES * 2 * BK * 4 + 4 * NSUB * OUT_BYTES + 1024;
  static constexpr uint32_t S_COL = 0, O_COL = NSUB * BK;      // tensor-memory columns
  // Instruction descriptor of kind::f16: D fp32 (1 at [4,6)), A and B bf16 (1 at [7,10), [10,13)), B MN-major (bit 16)
  // for the values, N >> 3 at [17,23), M >> 4 at [24,29).
  static constexpr uint32_t IDESC_QK = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BK >> 3) << 17) | (8u << 24);
  static constexpr uint32_t IDESC_PV_BF16 = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | (8u << 24);
  static constexpr uint32_t IDESC_PV_F16 = IDESC_PV_BF16 & ~((1u << 7) | (1u << 10));      // both fp16 (0)
};

// Shared-memory descriptors in the 128-byte swizzle (8 rows of 128 bytes make an atom of 1024): start >> 4 at [0,14),
// leading offset >> 4 at [16,30), stride offset >> 4 at [32,46), version 1 at [46,48), swizzle 2 at [61,64).
// K-major: the stride is from 8 rows to the next 8.  MN-major (values: rows are keys, 64 elements of the head
// to a row): the leading offset goes from 64 elements to the next 64, the stride from 8 keys to the next 8.
__device__ __forceinline__ uint64_t desc_of(uint32_t saddr, uint32_t leading) {
  return (uint64_t)((saddr >> 4) & 0x3FFF) | ((uint64_t)(leading >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// The whole warp comes by these, converged, and `leader` (one lane) issues: the operands then stay in uniform registers,
// which the instruction takes.  Behind a branch of one lane each would be moved there before every instruction
// (measured: 150 cycles from one to the next instead of the 64 that the product takes).
__device__ __forceinline__ void umma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t leader) {
  asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(leader) : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t leader) {
  asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc), "r"(leader) : "memory");
}
__device__ __forceinline__ void umma_commit(uint64_t* bar, uint32_t leader) {
  asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}"
               ::"r"(smem_u32(bar)), "r"(leader) : "memory");
}
__device__ __forceinline__ uint32_t elect_one() {               // one lane of a converged warp
  uint32_t pred;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(pred));
  return pred;
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Tensor memory with one row to a thread: 32 columns of it.
__device__ __forceinline__ void tmem_ld_row(uint32_t taddr, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_row(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
               : "memory");
}
__device__ __forceinline__ void tmem_st_row16(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
// Tensor memory in the layout of an mma.m16n8 result: 16 lanes (rows), a thread holds of every 8 columns the columns
// 2t, 2t + 1 of row g (registers 0, 1) and of row g + 8 (2, 3), g = lane / 4, t = lane % 4.  Against one row to a thread
// this leaves a thread a quarter of the columns, and so of the keys' scales, for four rows.
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float* r) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(taddr), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7])
               : "memory");
}
// ... and 4 columns of 32 bits (8 bf16 values) at a time: row g column t (register 0), row g + 8 (1).
__device__ __forceinline__ void tmem_st_p(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
template <int R>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool live) {   // 16 bytes to shared memory, zeros if !live
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p) : "memory"); }
// two fp32 operations to an instruction
__device__ __forceinline__ void mul2(float& a, float& b, float x, float y) {
  asm("{\n .reg .b64 u, v;\n mov.b64 u, {%0, %1};\n mov.b64 v, {%2, %3};\n mul.rn.f32x2 u, u, v;\n mov.b64 {%0, %1}, u;\n}"
      : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}
__device__ __forceinline__ void fma2(float& a, float& b, float x0, float x1, float y) {   // a = a * x0 + y, b = b * x1 + y
  asm("{\n .reg .b64 u, v, w;\n mov.b64 u, {%0, %1};\n mov.b64 v, {%2, %3};\n mov.b64 w, {%4, %4};\n fma.rn.f32x2 u, u, v, w;\n mov.b64 {%0, %1}, u;\n}"
      : "+f"(a), "+f"(b) : "f"(x0), "f"(x1), "f"(y));
}
__device__ __forceinline__ void add2(float& a, float& b, float x, float y) {
  asm("{\n .reg .b64 u, v;\n mov.b64 u, {%0, %1};\n mov.b64 v, {%2, %3};\n add.rn.f32x2 u, u, v;\n mov.b64 {%0, %1}, u;\n}"
      : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}

struct TilesParams {
  KvView c;
  BatchView b;
  AttnArgs a;
  AttnPlan p;                    // tiles: an upper bound over the whole batch
  float* part_o;
  float* part_lse;
  int* status;
  int rows_follow;               // the call's next launch is the other kernel, which reads nothing of this one's
  int items, few;                // sequences of up to `few` rows are another kernel's (0: none)
  uint32_t div_mul;              // r / group = (umulhi(r, div_mul) + r) >> div_shift for 0 <= r < 2^31
  int div_shift;
};
__device__ __forceinline__ int token_of(const TilesParams& p, int r) {
  return (int)((__umulhi((uint32_t)r, p.div_mul) + (uint32_t)r) >> p.div_shift);
}

// What scores are multiplied by.  A negative scale: the queries are negated.  Zero: a masked score, -infinity, has to stay one,
// so the smallest number above it, which takes the largest product to 5e-7.
__device__ __forceinline__ float score_scale(float scale_log2) { return fmaxf(fabsf(scale_log2), 0x1p-149f); }

// The grid has one thread block to an item, but a block that runs takes over blocks that have not started yet
// (clusterlaunchcontrol.try_cancel), item by item, so the items are dealt by who is about to be free, in the grid's order,
// without a counter in memory and without giving up shared or tensor memory in between.  One request per call; after one
// that found nothing there may be no other.
__device__ __forceinline__ void request_block(uint32_t answer, uint64_t* bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
               ::"r"(answer), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ bool taken_block(uint32_t answer, int& block) {
  uint32_t ok, x;
  asm volatile(
      "{\n .reg .pred p;\n .reg .b128 r;\n ld.shared.b128 r, [%2];\n clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n"
      " mov.u32 %1, 0;\n @p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n selp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok), "=r"(x) : "r"(answer) : "memory");
  block = (int)x;
  return ok != 0;
}
// One work item, as every role sees it.
struct Item {
  int b, head, split;
  int q0, past;                  // first row of the sequence in the call's tensors; its tokens before the call's
  int r0, n_rows;                // rows of the item, of the sequence
  int key0, key1;                // keys of the piece that any row sees
  int tiles;                     // of BK keys; -1: no more items
};
// The first tile of a causal item in which some row masks a key.
template <int D>
__device__ __forceinline__ int first_masked(const TilesParams& p, const Item& w) {
  return max(0, w.past + token_of(p, w.r0) + 1 - w.key0) / TileGeo<D>::BK;
}
// The whole warp takes part.  False: nothing to do.
template <int D>
__device__ __forceinline__ bool decode_item(const TilesParams& p, int item, int lane, Item& o) {
  using G = TileGeo<D>;
  o.split = item % p.p.splits;
  const int rest = item / p.p.splits;
  o.head = rest % p.c.n_kv_heads;
  const int tl = p.p.tiles - 1 - rest / p.c.n_kv_heads;        // later rows see more keys: they go first
  // which sequence the tl-th tile of the batch belongs to
  int before = 0, b = -1, mine = 0;
  for (int b0 = 0; b0 < p.b.n_seqs && b < 0; b0 += 32) {
    int n = 0;
    if (b0 + lane < p.b.n_seqs) {
      const int q0 = __ldg(p.b.q_start + b0 + lane), q1 = __ldg(p.b.q_start + b0 + lane + 1);
      // starts that make no sense have no tiles: those that there are (as many as the sound ones need) go to the others
      const bool sane = q0 >= 0 && q1 >= q0 && q1 <= p.b.tokens;
      if (!sane) report_device_error(p.status, HBL_ERR_RANGE);
      const long rows = sane ? (long)min(q1 - q0, p.b.max_q_len) * p.a.group : 0;
      n = rows > p.few ? (int)((rows + G::ROWS - 1) / G::ROWS) : 0;
    }
    int sum = n;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, sum, s);
      if (lane >= s) sum += x;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, before + sum > tl);
    if (hit) {
      const int l = __ffs(hit) - 1;
      b = b0 + l;
      mine = tl - before - (__shfl_sync(0xffffffffu, sum, l) - __shfl_sync(0xffffffffu, n, l));
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  if (b < 0) return false;
  o.b = b;
  SeqLens len;
  if (!sequence_lengths(p.b, b, p.c.page_shift, p.status, len)) return false;
  o.q0 = len.q0;
  o.past = len.kv - len.q_len;
  o.n_rows = min(len.q_len, p.b.max_q_len) * p.a.group;
  o.r0 = mine * G::ROWS;
  if (o.split > 0 && (long)o.split * p.p.chunk >= len.held) return false;
  const int last_tok = token_of(p, min(o.r0 + G::ROWS - 1, o.n_rows - 1));
  const int seen = p.a.causal ? max(0, min(len.held, o.past + last_tok + 1)) : len.held;
  o.key0 = o.split * p.p.chunk;
  o.key1 = o.split == p.p.splits - 1 ? seen : min(seen, o.key0 + p.p.chunk);
  o.tiles = o.key1 > o.key0 ? (o.key1 - o.key0 + G::BK - 1) / G::BK : 0;
  return true;
}

// 16-byte chunk c of row r in a tile of [columns of 64 elements][rows][128 bytes].
__device__ __forceinline__ uint32_t chunk_at(int r, int c, int half_bytes) {
  return (uint32_t)((c >> 3) * half_bytes + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}
__device__ __forceinline__ void store16(uint32_t saddr, const uint32_t (&w)[4]) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(saddr), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}

template <int BITS, int D>
__global__ void __launch_bounds__(kThreads, 1) attn_tiles_kernel(const __grid_constant__ TilesParams p) {
  using G = TileGeo<D>;
  constexpr int NSUB = G::NSUB, BK = G::BK, STAGES = G::STAGES;
  constexpr bool CODES = BITS < 16;
  // Registers of a thread by role: two softmax groups (one at head_dim 256), the producers, the rest; launched with 128
  // each, and what is taken must be given (2 SOFT + PROD + REST = 512).
  constexpr int SOFT = CODES ? 184 : 192, PROD = CODES ? 88 : 64, REST = CODES ? 56 : 64;
  static_assert(2 * SOFT + PROD + REST <= 512, "setmaxnreg waits for registers that nobody gives back");
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) uint64_t q_full, q_empty, k_full[STAGES], k_empty[STAGES], v_full[STAGES], v_empty[STAGES], s_full[NSUB], p_full[NSUB][2],
      o_full[NSUB], item_full[2], item_empty[2];
  __shared__ Item item_slot[2];
  __shared__ __align__(8) uint64_t steal_bar, near_end;
  __shared__ __align__(16) uint4 steal_answer;
  __shared__ __align__(16) uint32_t bad_scale[STAGES][4];       // keys of the tile whose value scale is not finite
  __shared__ float2 unit_of_tile[STAGES];                       // what the value scales are held against: now, and before / now
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag_s;
  volatile int* abort_flag = &abort_flag_s;
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~uintptr_t(1023));
  const uint32_t sq = smem_u32(base), sk = sq + NSUB * G::Q_BYTES, sv = sk + STAGES * G::KV_BYTES;
  float* scales = reinterpret_cast<float*>(base + (size_t)NSUB * G::Q_BYTES + (size_t)STAGES * 2 * G::KV_BYTES);   // [stage][2][BK]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wg = warp >> 2;

  if (threadIdx.x == 0) {
    mbar_init(&q_full, 64);
    mbar_init(&steal_bar, 1);
    mbar_init(&near_end, 1);
    for (int s = 0; s < 2; ++s) {
      mbar_init(&item_full[s], 1);
      mbar_init(&item_empty[s], 4 * NSUB + 4 + 1 + 2);          // warps that work on items
    }
    mbar_init(&q_empty, 1);
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&k_full[s], 128);
      mbar_init(&k_empty[s], CODES ? 1 + 4 * NSUB : 1);        // the last product that reads it, and every warp that read its scales
      mbar_init(&v_full[s], 128);
      mbar_init(&v_empty[s], 1);
    }
    for (int i = 0; i < NSUB; ++i) {
      mbar_init(&s_full[i], 1);
      for (int h = 0; h < 2; ++h) mbar_init(&p_full[i][h], 4);
      mbar_init(&o_full[i], 1);
    }
    abort_flag_s = 0;
    mbar_fence_init();
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  grid_dependency_wait();
  if (p.rows_follow) grid_launch_dependents();                 // what came before is complete: the other kernel may begin
  // The n-th item of this block, from the warp that looks them up (all lanes of the calling warp; false: gave up).
  auto next_item = [&](uint32_t n, Item& w) {
    const bool ok = __all_sync(0xffffffffu, mbar_wait(&item_full[n & 1], (n >> 1) & 1, abort_flag, p.status));
    if (ok) {
      w = item_slot[n & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(&item_empty[n & 1]);
    }
    return ok;
  };

  if (wg < NSUB) {
    // ------------------------------ softmax ------------------------------
    // bf16: one row to a thread.  Codes: four rows to a thread and a quarter of the columns (see tmem_ld64), because
    // every column comes with two scales from shared memory.  Measured: bf16 prompt of 8192 tokens 590 us with one
    // row, 627 with four; 512 queries over 16384 tokens at 8 bits 292 with one, 241 with four.
    regs_up<SOFT>();
    constexpr int R = CODES ? 4 : 1, NP = BK / 2 / R, NQ = BK / 32, NPQ = NP / NQ;     // rows; pairs of columns of a row: all, of 32 keys
    const int sub = wg, g = lane >> 2, t = R == 4 ? lane & 3 : 0, quad = warp & 3;
    const uint32_t lane_base = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t s_addr = lane_base + G::S_COL + sub * BK, o_addr = lane_base + G::O_COL + sub * D;
    constexpr uint32_t LOWER = 16u << 16;                      // rows 16 .. 31 of the warp
    auto at = [](int i, int q) { return R == 4 ? (i >> 1) * (BK / 2) + 4 * q + 2 * (i & 1) : 2 * q; };   // pair q of row i among the registers
    constexpr int STEP = R == 4 ? 8 : 2;                       // its columns: STEP q + 2t, + 1
    const float scale = score_scale(p.a.scale_log2);
    uint32_t it = 0, done = 0;                                 // tiles and items so far: barrier phases
    bool ok = true;
    for (uint32_t n = 0;; ++n) {
      if (!(ok = __all_sync(0xffffffffu, mbar_wait(&item_full[n & 1], (n >> 1) & 1, abort_flag, p.status)))) break;
      const Item& w = item_slot[n & 1];                        // kept until the end: registers are short here
      const int tiles = w.tiles, key0 = w.key0;
      if (tiles < 0) break;
      // the thread's rows: first + 8 i
      const int first = w.r0 + sub * 128 + quad * 32 + (R == 4 ? g : lane);
      auto limit = [&](int i) {                                // keys below it are seen by row i
        const int r = first + 8 * i;
        return r >= w.n_rows ? 0 : p.a.causal ? min(w.key1, w.past + token_of(p, r) + 1) : w.key1;
      };
      int low = 0x7fffffff;                                    // below it the warp masks nothing
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (first + 8 * i < w.n_rows) low = min(low, limit(i));
      low = __reduce_min_sync(0xffffffffu, low);
      float neg[R], l[R];                                      // minus the maximum so far (0: none yet, see `some`), p's sum
      uint32_t some = 0;                                       // rows that have seen a key
      float unit = 1.f;                                        // codes: O is in units of it
#pragma unroll
      for (int i = 0; i < R; ++i) { neg[i] = 0.f; l[i] = 0.f; }
      for (int j = 0; j < tiles; ++j, ++it) {
        const int k0 = key0 + j * BK;
        const int stage = it % STAGES;
        if (CODES && !(ok = __all_sync(0xffffffffu, mbar_wait(&k_full[stage], (it / STAGES) & 1, abort_flag, p.status)))) break;   // its scales
        if (!(ok = __all_sync(0xffffffffu, mbar_wait(&s_full[sub], it & 1, abort_flag, p.status)))) break;
        tc_fence_after();
        float x[BK];
        if constexpr (R == 4) {
#pragma unroll
          for (int h = 0; h < BK / 64; ++h) {
            tmem_ld64(s_addr + 64 * h, x + 32 * h);
            tmem_ld64(s_addr + LOWER + 64 * h, x + BK / 2 + 32 * h);
          }
        } else {
#pragma unroll
          for (int c = 0; c < BK / 32; ++c) tmem_ld_row(s_addr + 32 * c, x + 32 * c);
        }
        const float2* ks = reinterpret_cast<const float2*>(scales + stage * 2 * BK) + t;
        const float2* vs = ks + BK / 2;
        tmem_ld_wait();
        const bool masked = k0 + BK > low;
        // codes: scores relative to the maximum so far (bf16: the products alone, in units of which the mask and the
        // maximum are the same)
        if (CODES) {
#pragma unroll
          for (int q = 0; q < NP; ++q) {
            const float2 s = ks[4 * q];
#pragma unroll
            for (int i = 0; i < R; ++i) fma2(x[at(i, q)], x[at(i, q) + 1], s.x, s.y, neg[i]);
          }
        }
        if (masked) {
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const int seen = limit(i) - k0 - 2 * t;
#pragma unroll
            for (int q = 0; q < NP; ++q) {
              if (STEP * q >= seen) x[at(i, q)] = -INFINITY;
              if (STEP * q + 1 >= seen) x[at(i, q) + 1] = -INFINITY;
            }
          }
        }
        float top[R];                                           // how far the tile's largest score lies above the maximum
        bool raise = false;
#pragma unroll
        for (int i = 0; i < R; ++i) {
          constexpr int CHAINS = R == 4 ? 2 : 4;                // independent ones, to hide each operation's latency
          float c[CHAINS];
#pragma unroll
          for (int e = 0; e < CHAINS; ++e) c[e] = fmaxf(x[at(i, e)], x[at(i, e) + 1]);
#pragma unroll
          for (int q = CHAINS; q < NP; ++q) c[q % CHAINS] = fmaxf(c[q % CHAINS], fmaxf(x[at(i, q)], x[at(i, q) + 1]));
#pragma unroll
          for (int e = 1; e < CHAINS; ++e) c[0] = fmaxf(c[0], c[e]);
          top[i] = CODES ? c[0] : fmaf(c[0], scale, neg[i]);
          raise |= top[i] > (some >> i & 1 ? kLazy : -INFINITY);
        }
        float regauge = 1.f;
        if (CODES) {
          const float2 y = unit_of_tile[stage];
          unit = y.x;
          regauge = y.y;
          raise |= regauge != 1.f;
        }
        if (__any_sync(0xffffffffu, raise)) {
          float f[R];
#pragma unroll
          for (int i = 0; i < R; ++i) {
            if (R == 4) {
              top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
              top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
            }
            const bool old = some >> i & 1, up = top[i] > (old ? kLazy : -INFINITY);
            const float by = up ? top[i] : 0.f;                 // how far the maximum rises (from 0 where there was none)
            f[i] = up ? (old ? exp2_approx(-by) : 0.f) : 1.f;
            if (up) some |= 1u << i;
            neg[i] -= by;
            l[i] *= f[i];
            if (CODES) {
#pragma unroll
              for (int q = 0; q < NP; ++q) add2(x[at(i, q)], x[at(i, q) + 1], -by, -by);
            }
          }
          if (j > 0) {
#pragma unroll 1
            for (int c = 0; c < D / (R == 4 ? 16 : 32); ++c) {      // (few registers: the scores are held meanwhile)
              if constexpr (R == 4) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  float o[8];
                  tmem_ld16(o_addr + h * LOWER + 16 * c, o);
                  tmem_ld_wait();
#pragma unroll
                  for (int e = 0; e < 8; ++e) o[e] *= f[R == 4 ? 2 * h + (e >> 1 & 1) : 0] * regauge;
                  tmem_st16(o_addr + h * LOWER + 16 * c, o);
                }
              } else {
                float o[32];
                tmem_ld_row(o_addr + 32 * c, o);
                tmem_ld_wait();
                uint32_t u[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) u[e] = __float_as_uint(o[e] * f[0]);
                tmem_st_row(o_addr + 32 * c, u);
              }
            }
          }
        }
        float sum[R][4 / R > 1 ? 4 : 2] = {};
        // All but the last 32 keys are handed over first, so that their product runs while the rest is computed and the last
        // part's is short; the first hand-over, which waits for the stores, comes in the middle of the last part.
        auto hand_over = [&](int part) {
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&p_full[sub][part]);
        };
#pragma unroll
        for (int u = 0; u < NQ; ++u) {
          uint32_t pk[16];
#pragma unroll
          for (int c = 0; c < NPQ; ++c) {
            const int q = u * NPQ + c;
            const float2 v = CODES ? vs[4 * q] : make_float2(1.f, 1.f);
#pragma unroll
            for (int i = 0; i < R; ++i) {
              float y0 = x[at(i, q)], y1 = x[at(i, q) + 1];
              if (!CODES) fma2(y0, y1, scale, scale, neg[i]);
              y0 = exp2_approx(y0);
              y1 = exp2_approx(y1);
              const int chain = R == 4 ? 0 : 2 * (c & 1);
              add2(sum[i][chain], sum[i][chain + 1], y0, y1);
              if (CODES) mul2(y0, y1, v.x, v.y);
              pk[R == 4 ? (i >> 1) * 8 + 2 * c + (i & 1) : c] = CODES ? pack2_f16(y0, y1) : pack2(y0, y1);
            }
            if (u == NQ - 1 && c == NPQ / 2 - 1) hand_over(0);
          }
          if constexpr (R == 4) {
            tmem_st_p(s_addr + 16 * u, pk);
            tmem_st_p(s_addr + LOWER + 16 * u, pk + 8);
          } else {
            tmem_st_row16(s_addr + 16 * u, pk);
          }
        }
        hand_over(1);
#pragma unroll
        for (int i = 0; i < R; ++i) l[i] += R == 4 ? sum[i][0] + sum[i][1] : (sum[i][0] + sum[i][1]) + (sum[i][R == 4 ? 0 : 2] + sum[i][R == 4 ? 0 : 3]);
        if (CODES) {
          // a value scale that is not finite came as zero (0 * it would reach rows it is masked for): rows that see
          // its key are marked, and their results become NaN
          const uint4 b = *reinterpret_cast<const uint4*>(bad_scale[stage]);
          if (b.x | b.y | b.z | b.w) {
            const uint32_t word[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < R; ++i) {
              const int seen = limit(i) - k0;
              for (int e = 0; e < BK / 32; ++e) {
                const int n_seen = seen - 32 * e;
                if (word[e] & (n_seen <= 0 ? 0u : n_seen >= 32 ? ~0u : (1u << n_seen) - 1)) some |= 16u << i;
              }
            }
          }
          __syncwarp();                                         // every lane has read the stage's marks: lane 0 speaks for all
          if (lane == 0) mbar_arrive(&k_empty[stage]);
        }
      }
      if (!ok) break;
      // ---- the rows' results ----
      const bool whole = p.p.splits <= 1;
      float inv[R];
      char* mine[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (R == 4) {
          l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
          l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
        }
        inv[i] = l[i] == 0.f ? 0.f : __fdividef(unit, l[i]);
        if (some >> i & 16) inv[i] = __uint_as_float(0x7FC00000u);
        const int r = first + 8 * i;
        mine[i] = nullptr;
        if (r < w.n_rows) {
          const int tok = token_of(p, r), hq = w.head * p.a.group + r - tok * p.a.group;
          const long row = (long)(w.q0 + tok) * p.a.n_heads + hq, part = (long)w.split * p.b.tokens * p.a.n_heads + row;
          mine[i] = whole ? reinterpret_cast<char*>(p.a.out + (w.q0 + tok) * p.a.o_ts + hq * p.a.o_hs) : reinterpret_cast<char*>(p.part_o + part * D);
          const float lse2 = l[i] == 0.f ? -INFINITY : __log2f(l[i]) - neg[i];
          if (t == 0 && !whole) p.part_lse[part] = lse2;
          if (t == 0 && whole && p.a.lse != nullptr) p.a.lse[row] = lse2 * 0.6931471805599453f;
        }
      }
      // 64 bytes of every row at a time go by way of shared memory, where they get back into order and from where four
      // lanes write a row's together: this thread a quarter of the rows lane / 4 + 8 i
      char* dst[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        dst[i] = R == 4 ? mine[R == 4 ? i : 0]
                        : reinterpret_cast<char*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine[0]), 8 * i + g));
      const uint32_t out = smem_u32(scales + STAGES * 2 * BK) + (sub * 4 + quad) * G::OUT_BYTES;
      auto flush = [&](int byte) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t y[4];
          asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3])
                       : "r"(out + (8 * i + g) * G::OUT_PITCH + (lane & 3) * 16) : "memory");
          if (dst[i] != nullptr) *reinterpret_cast<uint4*>(dst[i] + byte + (lane & 3) * 16) = make_uint4(y[0], y[1], y[2], y[3]);
        }
        __syncwarp();
      };
      if (tiles > 0) {
        if (!(ok = __all_sync(0xffffffffu, mbar_wait(&o_full[sub], done & 1, abort_flag, p.status)))) break;
        ++done;
        tc_fence_after();
      }
      const int e0 = BITS == 8 ? 2 * t : t, e1 = BITS == 8 ? 2 * t + 1 : t + 4;
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        float o[32];
        if (tiles == 0) {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        } else if constexpr (R == 4) {
          tmem_ld32(o_addr + 32 * c, o);
          tmem_ld32(o_addr + LOWER + 32 * c, o + 16);
          tmem_ld_wait();
        } else {
          tmem_ld_row(o_addr + 32 * c, o);
          tmem_ld_wait();
        }
        if constexpr (R == 1) {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] *= inv[0];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (whole && h == 1) break;
            uint32_t u[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) u[e] = whole ? pack2(o[2 * e], o[2 * e + 1]) : __float_as_uint(o[16 * h + e]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t y[4] = {u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]};
              store16(out + lane * G::OUT_PITCH + 16 * i, y);
            }
            flush(whole ? 64 * c : 128 * c + 64 * h);
          }
        } else if (whole) {
          // a thread's columns 2t, 2t + 1 of each group of 8 are the head's elements e0, e1 of that group
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < R; ++i) {
              const float* y = &o[16 * (i >> 1) + 4 * q + 2 * (i & 1)];
              const uint32_t u = pack2(y[0] * inv[i], y[1] * inv[i]), a = out + (8 * i + g) * G::OUT_PITCH + 16 * q;
              asm volatile("st.shared.b16 [%0], %1;" ::"r"(a + 2 * e0), "h"((unsigned short)u) : "memory");
              asm volatile("st.shared.b16 [%0], %1;" ::"r"(a + 2 * e1), "h"((unsigned short)(u >> 16)) : "memory");
            }
          flush(64 * c);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
              for (int i = 0; i < R; ++i) {
                const float* y = &o[16 * (i >> 1) + 4 * (2 * h + q) + 2 * (i & 1)];
                const uint32_t a = out + (8 * i + g) * G::OUT_PITCH + 32 * q;
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(a + 4 * e0), "f"(y[0] * inv[i]) : "memory");
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(a + 4 * e1), "f"(y[1] * inv[i]) : "memory");
              }
            flush(128 * c + 64 * h);
          }
        }
      }
      tc_fence_before();                                        // O has been read: the next item's P says so to the issuer
      __syncwarp();
      if (lane == 0) mbar_arrive(&item_empty[n & 1]);
    }
  } else if (wg == 2) {
    // ------------------------------ producers ------------------------------
    regs_down<PROD>();
    const int tid = threadIdx.x & 127;
    constexpr int CH = D / 8;                                   // 16-byte chunks of a row
    const float scale = score_scale(p.a.scale_log2);
    uint32_t it = 0;
    bool ok = true;
    Item w;
    for (uint32_t n = 0; ok && (ok = next_item(n, w)) && w.tiles >= 0; ++n) {
      if (w.tiles == 0) continue;
      const int* page_row = p.b.pages + (long)w.b * p.b.max_pages;
      // pages of a tile's 16-key groups, one to a lane (a tile starts on a multiple of 64 keys; a group lies in one page)
      auto page_of = [&](int j) {
        const int key = w.key0 + j * BK + 16 * lane;
        return lane < BK / 16 && key < w.key1 ? __ldg(page_row + (key >> p.c.page_shift)) : -1;
      };
      struct Tile { long group_row; unsigned good; int there; };
      auto open = [&](int j, int page) {
        const int k0 = w.key0 + j * BK;
        const bool in = page >= 0 && page < p.c.n_pages;
        if (lane < BK / 16 && k0 + 16 * lane < w.key1 && !in) report_device_error(p.status, HBL_ERR_RANGE);
        Tile t;
        t.group_row = cache_row(p.c, in ? page : 0, w.head, (k0 + 16 * lane) & ((1 << p.c.page_shift) - 1));
        t.good = __ballot_sync(0xffffffffu, in);
        t.there = w.key1 - k0;                                  // keys of the tile that exist
        return t;
      };
      auto row_of = [&](const Tile& t, int rr) { return __shfl_sync(0xffffffffu, t.group_row, rr >> 4) + (rr & 15); };
      auto live = [&](const Tile& t, int rr) { return rr < t.there && (t.good >> (rr >> 4) & 1); };
      int next_page = page_of(0);
      Tile tile = open(0, next_page);
      next_page = page_of(1);
      if constexpr (!CODES) {
        // bf16 rows are copied asynchronously and announced one copy later, so that two are in flight; nothing that a
        // wait below needs depends on the one not announced yet
        uint64_t* copied = nullptr;
        const int masked_from = p.a.causal ? first_masked<D>(p, w) : w.tiles;
        for (int j = 0; j < w.tiles; ++j, ++it) {
          const int stage = it % STAGES;
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            uint64_t* empty = kv == 0 ? &k_empty[stage] : &v_empty[stage];
            if (!(ok = __all_sync(0xffffffffu, mbar_wait<true>(empty, ((it / STAGES) & 1) ^ 1, abort_flag, p.status)))) break;
            const uint32_t dst = (kv == 0 ? sk : sv) + stage * G::KV_BYTES;
            const unsigned char* col = (kv == 0 ? p.c.k : p.c.v) + (tid % CH) * 16;
            constexpr int RPP = 128 / CH;                       // rows side by side
#pragma unroll
            for (int i = 0; i < BK / RPP; ++i) {
              const int rr = i * RPP + tid / CH;
              copy16(dst + chunk_at(rr, tid % CH, G::HALF), col + row_of(tile, rr) * (2 * D), live(tile, rr));
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (kv == 1 && j >= masked_from) {
              // A tile that some row masks: 0 * a value that is not finite would reach rows that mask its key.  Every thread
              // looks through the pieces that it has copied; such a key's value becomes zeros and the key itself NaN, so
              // that the rows that see it, and no others, become NaN.  (The same lanes hold a row's pieces of both.)
              asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll 2
              for (int i = 0; i < BK / RPP; ++i) {
                const uint32_t at = chunk_at(i * RPP + tid / CH, tid % CH, G::HALF);
                uint32_t y[4], sum = 0;                         // 0 * y: zeros, or NaN where y is not finite
                asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]) : "r"(dst + at) : "memory");
#pragma unroll
                for (int k = 0; k < 4; ++k) asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(y[k]), "r"(0u));
                const unsigned bad = __ballot_sync(0xffffffffu, (sum & 0x7FFF7FFFu) != 0);
                if (bad >> (lane & ~(CH - 1)) & (CH == 32 ? ~0u : (1u << CH % 32) - 1)) {
                  const uint32_t zero[4] = {0, 0, 0, 0}, nan[4] = {0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
                  store16(dst + at, zero);
                  store16(sk + stage * G::KV_BYTES + at, nan);
                }
              }
              fence_async();
              mbar_arrive(copied);                              // the keys
              mbar_arrive(&v_full[stage]);
              copied = nullptr;
              continue;
            }
            if (copied != nullptr) {
              asm volatile("cp.async.wait_group 1;" ::: "memory");
              fence_async();                                    // what the copies wrote is read next by the tensor cores
              mbar_arrive(copied);
            }
            copied = kv == 0 ? &k_full[stage] : &v_full[stage];
          }
          if (!ok) break;
          if (j + 1 < w.tiles) {
            tile = open(j + 1, next_page);
            next_page = page_of(j + 2);
          }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (ok && copied != nullptr) {
          fence_async();
          mbar_arrive(copied);
        }
      } else {
        int bos_row = -1;
        if (BITS < 8 && p.c.bos_k != nullptr && w.key0 == 0) {
          const int slot = p.b.bos_slot != nullptr ? __ldg(p.b.bos_slot + w.b) : w.b;
          if (slot >= 0 && slot < p.c.n_slots) bos_row = slot;
          else if (tid == 0) report_device_error(p.status, HBL_ERR_RANGE);
        }
        // A lane widens UN units (UN * BITS bytes) of a row; BATCH rows of it are loaded while the batch before is
        // widened, across tiles.
        constexpr int UN = BITS == 8 ? 2 : 4, LPR = D / 8 / UN, RPP = 128 / LPR, PASSES = BK / RPP;
        constexpr int BATCH = PASSES < 4 ? PASSES : 4, NB = PASSES / BATCH;
        // Eight neighbouring lanes take pieces of the same 64 elements of UN rows: their 16-byte stores then fall into
        // eight different bank groups of the swizzle.
        constexpr int PH = 8 / UN, HALVES = D / 64;
        const int piece = tid / 8 % HALVES * PH + tid % PH, my_row = tid / (8 * HALVES) * UN + tid / PH % UN;
        using L1 = Lane<BITS, UN, LPR>;
        static_assert(L1::UPC == UN && PASSES % BATCH == 0, "one piece of a row to a lane, whole batches");
        struct Raw { L1 r[BATCH]; };
        auto load = [&](Raw& raw, const Tile& t, int kv, int batch) {
          const unsigned char* src = kv == 0 ? p.c.k : p.c.v;
#pragma unroll
          for (int i = 0; i < BATCH; ++i) {
            const int rr = (batch * BATCH + i) * RPP + my_row;
            raw.r[i].load(src + row_of(t, rr) * (D * BITS / 8), piece, live(t, rr));
          }
        };
        // Scales: ks of key row tid; value scales of all rows (32 i + lane), so that every warp finds the same `unit`
        // for itself: a power of two no smaller than any value scale of the item so far.  p vs / unit * 2^7 is at most
        // 2^15, what fp16 holds; it is rounded by 2^-11 of itself, or by 2^-32 unit where it is that small.
        constexpr int VN = BK / 32;
        float ks = 0.f, vs[VN];
        auto load_scales = [&](const Tile& t) {
#pragma unroll
          for (int i = 0; i < VN; ++i) {
            const long row = row_of(t, 32 * i + lane);
            vs[i] = live(t, 32 * i + lane) ? __ldg(p.c.v_scale + row) : 0.f;
          }
          if (tid < BK) {                                       // (whole warps)
            const long row = row_of(t, tid);
            ks = live(t, tid) ? __ldg(p.c.k_scale + row) : 0.f;
          }
        };
        float unit = 0x1p-100f;
        Raw raw, ahead;
        load(raw, tile, 0, 0);
        load_scales(tile);
        for (int j = 0; j < w.tiles; ++j, ++it) {
          const int stage = it % STAGES;
          const bool special = BITS < 8 && w.key0 + j == 0 && p.c.bos_k != nullptr, more = j + 1 < w.tiles;
          Tile after = tile;
          if (more) after = open(j + 1, next_page);
          next_page = page_of(j + 2);
          if (more && tid < BK) {                               // the next tile's rows towards L2 (a row: 32 .. 256 bytes)
            const long row = row_of(after, tid) * (D * BITS / 8);
            if (live(after, tid)) {
#pragma unroll
              for (int b = 0; b < D * BITS / 8; b += 128) {
                prefetch_l2(p.c.k + row + b);
                prefetch_l2(p.c.v + row + b);
              }
            }
          }
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const uint32_t dst = (kv == 0 ? sk : sv) + stage * G::KV_BYTES;
            uint64_t* empty = kv == 0 ? &k_empty[stage] : &v_empty[stage];
#pragma unroll
            for (int batch = 0; batch < NB; ++batch) {
              if (batch + 1 < NB) load(ahead, tile, kv, batch + 1);
              else if (kv == 0) load(ahead, tile, 1, 0);
              else if (more) load(ahead, after, 0, 0);
              if (batch == 0) {
                if (!(ok = __all_sync(0xffffffffu, mbar_wait<true>(empty, ((it / STAGES) & 1) ^ 1, abort_flag, p.status)))) break;
                if (kv == 0) {
                  // scales of both with the keys: ks_j * sm_scale * log2(e), vs_j / unit * 2^7
                  if (special && lane == 0) {
                    const long brow = (long)bos_row * p.c.n_kv_heads + w.head;
                    if (tid == 0) ks = bos_row >= 0 ? __ldg(p.c.bos_k_scale + brow) : 0.f;
                    vs[0] = bos_row >= 0 ? __ldg(p.c.bos_v_scale + brow) : 0.f;
                  }
                  uint32_t most = 0, bad = 0;
#pragma unroll
                  for (int i = 0; i < VN; ++i) {
                    const uint32_t x = __float_as_uint(fabsf(vs[i]));
                    if (x >= 0x7F800000u) {
                      bad |= 1u << i;
                      vs[i] = 0.f;
                    } else {
                      most = max(most, min(x, 0x7E800000u));
                    }
                  }
                  const float before = unit;
                  unit = fmaxf(unit, __uint_as_float((__reduce_max_sync(0xffffffffu, most) + 0x7FFFFFu) & 0x7F800000u));
                  const float to = 128.f / unit;
                  const int mine = tid >> 5;                     // of the tile's 32-key groups
                  float my_vs = 0.f;
#pragma unroll
                  for (int i = 0; i < VN; ++i)
                    if (i == mine) my_vs = vs[i];
                  const unsigned word = __ballot_sync(0xffffffffu, mine < VN && (bad >> mine & 1));
                  if (lane == 0) bad_scale[stage][mine] = word;  // (BK 64: the upper two hold none)
                  if (tid == 0) unit_of_tile[stage] = make_float2(unit * 0x1p-7f, before / unit);
                  if (tid < BK) {
                    scales[stage * 2 * BK + tid] = ks * scale;
                    scales[stage * 2 * BK + BK + tid] = my_vs * to;
                  }
                  if (more) load_scales(after);
                }
              }
#pragma unroll
              for (int i = 0; i < BATCH; ++i) {
                const int rr = (batch * BATCH + i) * RPP + my_row;
                if (special && rr == 0) continue;
#pragma unroll
                for (int u = 0; u < UN; ++u) {
                  uint32_t o[4];
                  if (kv == 0) pairs<BITS>(raw.r[i], u, piece, o);
                  else pairs16<BITS>(raw.r[i], u, piece, o);
                  store16(dst + chunk_at(rr, piece * UN + u, G::HALF), o);
                }
              }
              raw = ahead;
            }
            if (!ok) break;
            if (special && tid < CH) {                          // the first token's row from its 8-bit codes
              uint32_t o[4] = {0, 0, 0, 0};
              if (bos_row >= 0) {
                const long brow = (long)bos_row * p.c.n_kv_heads + w.head;
                const uint2 u = __ldg(reinterpret_cast<const uint2*>((kv == 0 ? p.c.bos_k : p.c.bos_v) + brow * D) + tid);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  auto value = [&](int e) { return (float)((int)(((e < 4 ? u.x : u.y) >> (8 * (e & 3))) & 255u) - 128); };
                  o[k] = kv == 0 ? pack2(value(pair_lo<BITS>(k)), value(pair_hi<BITS>(k))) : pack2_f16(value(pair16_lo<BITS>(k)), value(pair16_hi<BITS>(k)));
                }
              }
              store16(dst + chunk_at(0, tid, G::HALF), o);
            }
            fence_async();                                      // generic-proxy writes, read next by the tensor cores
            mbar_arrive(kv == 0 ? &k_full[stage] : &v_full[stage]);
          }
          if (!ok) break;
          tile = after;
        }
      }
    }
  } else if (wg == 3) {
    // ------------------------------ issuer, the queries, the items ------------------------------
    regs_down<REST>();
    if (warp == 12) {
      const uint32_t leader = elect_one();
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      const uint64_t qd = desc_of(sq, 16), kd = desc_of(sk, 16), vd = desc_of(sv, G::HALF);
      uint32_t it = 0, items = 0;
      bool ok = true;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        ok = __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, p.status));
        tc_fence_after();
        return ok;
      };
      auto scores = [&](int i, uint32_t stage) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          umma_ss(tm + G::S_COL + i * BK, qd + (uint64_t)((i * G::Q_BYTES + (k >> 2) * (128 * 128) + (k & 3) * 32) >> 4),
                  kd + (uint64_t)((stage * G::KV_BYTES + (k >> 2) * G::HALF + (k & 3) * 32) >> 4), G::IDESC_QK, k != 0, leader);
        umma_commit(&s_full[i], leader);
      };
      Item w;
      for (uint32_t n = 0; ok && (ok = next_item(n, w)) && w.tiles >= 0; ++n) {
        if (w.tiles == 0) {
          if (lane == 0) mbar_arrive(&near_end);
          continue;
        }
        if (!wait(&q_full, items & 1) || !wait(&k_full[it % STAGES], (it / STAGES) & 1)) break;
        ++items;
#pragma unroll
        for (int i = 0; i < NSUB; ++i) scores(i, it % STAGES);
        umma_commit(&k_empty[it % STAGES], leader);
        if (w.tiles == 1) umma_commit(&q_empty, leader);
        for (int j = 0; j < w.tiles; ++j, ++it) {
          const uint32_t stage = it % STAGES, next = (it + 1) % STAGES;
          const bool more = j + 1 < w.tiles;
          if (j == max(0, w.tiles - kNearEnd) && lane == 0) mbar_arrive(&near_end);
          if (!wait(&v_full[stage], (it / STAGES) & 1)) break;
#pragma unroll
          for (int i = 0; i < NSUB; ++i) {
#pragma unroll
            for (int k = 0; k < BK / 16; ++k) {
              if ((k == 0 || k == BK / 16 - 2) && !wait(&p_full[i][k != 0], it & 1)) break;
              umma_ts(tm + G::O_COL + i * D, tm + G::S_COL + i * BK + 8 * k, vd + (uint64_t)((stage * G::KV_BYTES + k * 2048) >> 4),
                      CODES ? G::IDESC_PV_F16 : G::IDESC_PV_BF16, (j | k) != 0, leader);
            }
            if (!ok) break;
            if (more) {
              if (i == 0 && !wait(&k_full[next], ((it + 1) / STAGES) & 1)) break;
              scores(i, next);
            } else {
              umma_commit(&o_full[i], leader);
            }
          }
          if (!ok) break;
          umma_commit(&v_empty[stage], leader);
          if (more) umma_commit(&k_empty[next], leader);
          if (j + 2 == w.tiles) umma_commit(&q_empty, leader);   // the item's last scores: its queries may go
        }
      }
    }
    if (warp == 15) {
      // ---- the items.  The next one is asked for when the last tiles of the one before are at work: early enough to be
      // there in time with its queries, and not earlier, because a block that holds an item that it cannot begin keeps it
      // from those that are free ----
      uint32_t made = 0;
      bool ok = true;
      auto give = [&](const Item& w) {
        ok = __all_sync(0xffffffffu, mbar_wait<true>(&item_empty[made & 1], ((made >> 1) & 1) ^ 1, abort_flag, p.status));
        if (ok && lane == 0) {
          item_slot[made & 1] = w;
          mbar_arrive(&item_full[made & 1]);
        }
        ++made;
      };
      Item w;
      int item = blockIdx.x;
      for (uint32_t n = 0; ok; ++n) {
        if (decode_item<D>(p, item, lane, w)) {
          give(w);
          // (a long wait, which the softmax warp beside this one should not notice)
          for (int i = 0; ok && i < 1000000 && !mbar_try(&near_end, (made - 1) & 1) && !*abort_flag; ++i) __nanosleep(500);
          if (!ok || !(ok = __all_sync(0xffffffffu, mbar_wait<true>(&near_end, (made - 1) & 1, abort_flag, p.status)))) break;
        }
        if (lane == 0) {
          mbar_expect_tx(&steal_bar, 16);
          request_block(smem_u32(&steal_answer), &steal_bar);
        }
        if (!(ok = __all_sync(0xffffffffu, mbar_wait<true>(&steal_bar, n & 1, abort_flag, p.status)))) break;
        const bool more = taken_block(smem_u32(&steal_answer), item);
        fence_async();                                          // the answer has been read before the next one is written
        __syncwarp();
        if (!more) break;
      }
      w.tiles = -1;
      if (ok) give(w);
    } else if (warp > 12) {
      // ---- queries: as soon as the last scores of the item before are done, while its last products still run ----
      constexpr int CH = D / 8, RPP = 64 / CH, N = NSUB * 128;
      const int tid = threadIdx.x - 13 * 32;
      const bool reorder = CODES || p.a.scale_log2 < 0.f;
      const uint32_t flip = p.a.scale_log2 < 0.f ? 0x80008000u : 0u;
      uint32_t items = 0;
      bool ok = true;
      Item w;
      for (uint32_t n = 0; ok && (ok = next_item(n, w)) && w.tiles >= 0; ++n) {
        if (w.tiles == 0) continue;
        if (!(ok = __all_sync(0xffffffffu, mbar_wait<true>(&q_empty, (items & 1) ^ 1, abort_flag, p.status)))) break;
        ++items;
        const int c = tid % CH, first = tid / CH, step_tok = token_of(p, RPP), step_rem = RPP - step_tok * p.a.group;
        const int tok0 = token_of(p, w.r0 + first);
        int rem = w.r0 + first - tok0 * p.a.group;
        const __nv_bfloat16* q = p.a.q + w.q0 * p.a.q_ts + (long)w.head * p.a.group * p.a.q_hs + 8 * c;
        const __nv_bfloat16* from = q + tok0 * p.a.q_ts + rem * p.a.q_hs;
        // from one row to the next that is this thread's: over whole tokens, and back by a token's heads where they end
        const long ahead = step_tok * p.a.q_ts + step_rem * p.a.q_hs, back = p.a.q_ts - p.a.group * p.a.q_hs;
        const int there = w.n_rows - w.r0;
#pragma unroll 8
        for (int i = 0; i < N / RPP; ++i) {
          const int rr = first + RPP * i;
          const bool live = rr < there;
          copy16(sq + (rr >> 7) * G::Q_BYTES + chunk_at(rr & 127, c, 128 * 128), live ? from : q, live);
          from += ahead;
          rem += step_rem;
          if (rem >= p.a.group) {
            rem -= p.a.group;
            from += back;
          }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (reorder)                                            // each thread its own pieces
          for (int rr = first; rr < N; rr += RPP) {
            const uint32_t at = sq + (rr >> 7) * G::Q_BYTES + chunk_at(rr & 127, c, 128 * 128);
            uint32_t y[4], o[4];
            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]) : "r"(at) : "memory");
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int lo = pair_lo<BITS>(k), hi = pair_hi<BITS>(k);
              o[k] = __byte_perm(y[lo / 2], y[hi / 2], (lo & 1 ? 0x32 : 0x10) | (hi & 1 ? 0x7600 : 0x5400)) ^ flip;
            }
            store16(at, o);
          }
        fence_async();
        mbar_arrive(&q_full);
      }
    }
  } else {
    regs_down<REST>();                                            // (head_dim 256: the second softmax group has no sub-tile)
  }

  // ------------------------------ teardown ------------------------------
  __syncwarp();
  if (*abort_flag) {                                            // products in flight may still read shared memory
    const uint64_t t0 = global_ns();
    while (global_ns() - t0 < 200000ull) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 12) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

template <int BITS, int D>
int launch_tiles_dim(TilesParams& p, cudaStream_t s) {
  auto kern = attn_tiles_kernel<BITS, D>;
  HBL_ALLOW_DYNAMIC_SMEM(kern, TileGeo<D>::SMEM);
  HBL_CUDA_OK(launch_waiting(kern, dim3(p.items), dim3(kThreads), TileGeo<D>::SMEM, s, p));
  note_launch();
  return HBL_OK;
}
template <int BITS>
int launch_tiles_bits(TilesParams& p, cudaStream_t s) {
  switch (p.c.head_dim) {
    case 64: return launch_tiles_dim<BITS, 64>(p, s);
    case 128: return launch_tiles_dim<BITS, 128>(p, s);
    case 256: return launch_tiles_dim<BITS, 256>(p, s);
    default: return HBL_ERR_SHAPE;
  }
}

}  // namespace

AttnPlan plan_attention_tiles(const KvView& c, const BatchView& b, int n_heads, int few) {
  AttnPlan p{};
  const int group = n_heads / c.n_kv_heads, rows = c.head_dim == 256 ? 128 : 256;
  // Whole tiles of all sequences together, and a partial one for each that has more than `few` rows.
  const long all = (long)b.tokens * group;
  const long partial = all / (few + 1) < b.n_seqs ? all / (few + 1) : b.n_seqs;
  long tiles = all / rows + partial;
  const long by_seq = (long)b.n_seqs * (((long)b.max_q_len * group + rows - 1) / rows);
  if (by_seq < tiles) tiles = by_seq;
  p.tiles = (int)(tiles < 0x7fffffffL ? tiles : 0x7fffffffL);
  const long base = tiles * c.n_kv_heads;
  // pieces of at least 1024 keys while there are fewer items than SMs, and of at most 2^24 (131072 tiles, some 0.3 s): the
  // kernel's bounded waits, of 2 s, last as long as an item
  const long want = base > 0 && base < sm_count() ? sm_count() / base : 1;
  const long most = ((long)b.max_kv_len + 1023) / 1024, least = ((long)b.max_kv_len + (1L << 24) - 1) >> 24;
  long n = want < most ? want : most;
  if (n < least) n = least;
  if (n < 1) n = 1;
  p.chunk = (int)((((long)b.max_kv_len + n - 1) / n + 127) / 128 * 128);
  if (p.chunk < 128) p.chunk = 128;
  p.splits = (int)(((long)b.max_kv_len + p.chunk - 1) / p.chunk);
  if (p.splits < 1) p.splits = 1;
  return p;
}

int launch_attention_tiles(const KvView& c, const BatchView& b, const AttnArgs& a, const AttnPlan& plan, int few, const AttnParts& w,
                           cudaStream_t s) {
  TilesParams p{};
  p.c = c; p.b = b; p.a = a; p.p = plan; p.few = few; p.part_o = w.tiles_o; p.part_lse = w.tiles_lse; p.rows_follow = few > 0;
  p.status = device_status_word();
  if (p.status == nullptr) return HBL_ERR_CUDA;
  const long items = (long)plan.tiles * c.n_kv_heads * plan.splits;
  if (items > 0x7fffffffL - 65536) return HBL_ERR_TOO_LARGE;
  p.items = (int)items;
  while ((1 << p.div_shift) < a.group) ++p.div_shift;
  p.div_mul = (uint32_t)(((((uint64_t)1 << p.div_shift) - a.group) << 32) / a.group + 1);
  switch (c.bits) {
    case 3: return launch_tiles_bits<3>(p, s);
    case 4: return launch_tiles_bits<4>(p, s);
    case 8: return launch_tiles_bits<8>(p, s);
    case 16: return launch_tiles_bits<16>(p, s);
    default: return HBL_ERR_BITS;
  }
}

}  // namespace hbl
