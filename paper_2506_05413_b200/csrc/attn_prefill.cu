// Attention over packed prompts of different lengths: queries [total_q] and keys [total_k] of all sequences one after
// another, grouped heads, causal (aligned at the sequences' ends) or not.
//
//   y_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = 2^(c q_i.k_j - m_i),  c = scale log2(e),  j <= i + keys - queries where causal
//
// in one pass over the keys with a running reference m_i.  Both products run on the fifth-generation tensor
// cores with their accumulators in tensor memory, a block of 64 keys at a time:
//
//   S = Q K^T    A = 128 query rows (shared memory), B = 64 keys, D = 64 fp32 columns of tensor memory
//   O += P V     A = P, the weights as fp16 in tensor memory (over S, which is done with), B = V as it
//                lies in memory (rows of keys: the MN-major form), D = head_dim fp32 columns
//
// A CTA owns two tiles of 128 query rows of one key head.  The rows of a tile are the heads of the
// group for one token after another, so that grouped heads share every key and value that is
// loaded, and a short prompt fills a tile.  A tile has two score buffers: the scores of block j + 2 are computed as soon
// as the weights of block j are used up, while the softmax works on block j + 1.  Two tiles with their two buffers
// and their outputs are all 512 columns of tensor memory.
//
// A thread of the softmax warps owns one row: its 64 scores come into registers with tcgen05.ld,
// so maximum and sum need no exchange.  The reference m is set 7 below the row's maximum and raised only when a maximum
// exceeds it by more than 15: then the row of O is multiplied down in tensor memory, which happens in the first few blocks
// and hardly ever after.  Sums, scores, O and m are fp32; a weight is rounded once to fp16, the type of the values that it
// multiplies.  It is at most 2^15 and keeps its 11 bits down to 2^-21 of the row's largest, and counts down to 2^-31: small
// weights add up over a long prompt.
//
// Roles: warps 0-3 and 4-7 the softmax of the two tiles, warps 8 and 9 issue their products, warp 10 the TMA
// loads (queries, then keys and values through one ring), warp 11 cleans the value rows that not every row
// of the CTA sees: a product of a zero weight with NaN or infinity is NaN, so rows past the sequence's end are
// zeroed, and values that are not finite taken out of causally masked blocks and put back, row by row, at the end.
// Every mbarrier wait is bounded; on expiry the CTA records a code and winds down.
//
// Measured (32 query heads, 8 key heads, head width 128, causal): a prompt of 8192 tokens, 550 GFLOP, 519-530 us in graph replays
// of milliseconds (1.04 to 1.06 PFLOP/s) and 565 to 609 in repeated calls over tenths of a second, where the power cap
// lowers the clock (0.90 to 0.97); 9 prompts of 2048 tokens in all with prefixes 31 to 33 us.  A block takes a tile 1900 cycles of
// 1.85 GHz.  What bounds it is that tile's chain: the thread that issues a tile's 12 products and waits and commits for them is busy for
// all of that (shared memory serves the operands, 192 bytes a cycle wanted with 64 keys a product, 128 given, and is slow to
// answer barriers beside that), and the softmax's 1150 cycles and the two waits for scores lie beside it.  Of an
// earlier 531 us it was 492 without the exponentials, 510 without the softmax's arithmetic, 482 with an eighth of the
// products.  Not better: the weights of 128 keys handed over in halves (686), two threads per row (577), one product warp for both
// tiles (898), 2^x by polynomial for some of the pairs (531 and up).  128 keys at a time with one buffer was 560 with one product
// warp and a descriptor worked out for every product; with the present issue of products it has not been measured.  Beside
// its blocks a CTA costs some 6 us, which is what a short prompt pays: 860 ns between two CTAs on an SM, 1900 cycles to set up,
// 3500 until the first scores, 2000 to 3000 from the last weights to the output, 3600 for the output (7 us in all with every thread storing its own
// row).  A CTA that takes on the work of CTAs that have not started (clusterlaunchcontrol) and loads ahead saves the first three, but
// its output needs room of its own, and the ring's fifth entry is worth as much: 34.2 and 543 us.
#include <cuda.h>

#include "common.cuh"
#include "rowquant.cuh"

namespace smoothrot {
namespace prefill {

constexpr int kRange = 35;
enum Site { kSiteLoad = 36, kSiteMma = 37, kSiteSoftmax = 38, kSiteGuard = 39, kSiteOutput = 40 };
constexpr unsigned long long kWaitLimitNs = 2000000000ull;
constexpr unsigned long long kDrainNs = 50000ull;
constexpr unsigned long long kAtOnceNs = 1000;   // a limit below this: the loads give up before the first copy (for tests)

__device__ int g_prefill_status = 0;
__device__ unsigned long long g_prefill_wait_limit_ns = kWaitLimitNs;

constexpr int kTile = 128;         // query rows of a tile
constexpr int kBlock = 64;         // keys of a block
constexpr int kRaggedBlocks = 6;   // of a CTA: its rows are at most 256 tokens, so 5 blocks in which they see different keys
constexpr int kThreads = 384;
constexpr int kSoftmaxWarps = 8;   // 4 a tile, a thread per row
constexpr int kMmaWarp = kSoftmaxWarps, kLoadWarp = kMmaWarp + 2, kGuardWarp = kLoadWarp + 1;      // a product warp per tile
constexpr int kGuardThreads = 32;
constexpr float kLead = 7.0f, kHeadroom = 15.0f;   // log2 of a row's largest weight when its reference is set, and at most

template <int D>
struct Cfg {
  static constexpr int kAtoms = D / 64;                       // 128-byte wide slices of a row
  static constexpr int kAtomBytes = kTile * 128;
  static constexpr int kTileBytes = kAtoms * kAtomBytes;      // 128 rows of queries
  static constexpr int kSliceBytes = kBlock * 128;
  static constexpr int kBlockBytes = kAtoms * kSliceBytes;    // 64 rows of keys or values
  static constexpr int kStages = D == 128 ? 5 : 8;            // of the ring: two blocks each
  static constexpr int kBarriers = 2 * kStages + 4 /*S*/ + 4 /*P*/ + 2 /*O*/ + 1 /*Q*/ + 2 * kRaggedBlocks;
  static constexpr int kBarOffset = 2 * kTileBytes + kStages * 2 * kBlockBytes;
  static constexpr int kMiscOffset = kBarOffset + 8 * kBarriers;
  static constexpr int kSmemBytes = kMiscOffset + 256;
  static_assert(kSmemBytes <= 227 * 1024, "shared memory budget");
};

struct Args {
  const __half* v;
  int64_t ldv, ldy;
  __half* y;
  int64_t total_q, total_k;
  const int32_t *cu_q, *cu_k;
  int batch, group, causal;
  int heads_per_chunk;       // heads of a group that a CTA handles: all, up to 128
  int chunks;                // of a group
  int tokens;                // per tile: 128 / heads_per_chunk
  int units;                 // kv heads * chunks
  float c;                   // |scale| log2(e), 1 where scale is 0
  int sign;                  // of scale: scores are multiplied by it
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// Bounded wait on a phase; false if it ran out or another role of the CTA gave up.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int site) {
  if (mbar_try(bar, parity)) return true;
  const unsigned long long t0 = now_ns();
  for (uint32_t spin = 1;; ++spin) {
    if (mbar_try(bar, parity)) return true;
    if ((spin & 63u) == 0u) {
      if (*abort_flag != 0) return false;
      if (now_ns() - t0 > g_prefill_wait_limit_ns) {
        *abort_flag = 1;
        atomicCAS(&g_prefill_status, 0, site);
        return false;
      }
    }
  }
}
// The same for a whole warp, with one answer for all of its lanes: what follows has instructions of the whole warp.
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag, int site) {
  constexpr uint32_t all = 0xffffffffu;
  if (__all_sync(all, mbar_try(bar, parity))) return true;
  const unsigned long long t0 = now_ns();
  for (uint32_t spin = 1;; ++spin) {
    if (__all_sync(all, mbar_try(bar, parity))) return true;
    if ((spin & 63u) == 0u) {
      const bool late = now_ns() - t0 > g_prefill_wait_limit_ns;
      if (__any_sync(all, late || *abort_flag != 0)) {
        if (late) {
          *abort_flag = 1;
          atomicCAS(&g_prefill_status, 0, site);
        }
        return false;
      }
    }
  }
}

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// K-major operand, 128-byte swizzle: rows of 128 bytes, groups of 8 rows 1024 bytes apart.
// Only the low word differs from one descriptor to the next: the address in 16 bytes, and the second stride above it.
__device__ __forceinline__ uint32_t desc_k_major(uint32_t addr) { return ((addr & 0x3FFFFu) >> 4) | (1u << 16); }
// MN-major operand, 128-byte swizzle: 64 values of N per 128-byte row, one row per k, groups of 8 k
// 1024 bytes apart, the next 64 values of N one slice of 64 rows further.
__device__ __forceinline__ uint32_t desc_mn_major(uint32_t addr) {
  return ((addr & 0x3FFFFu) >> 4) | ((uint32_t(kBlock) * 128u >> 4) << 16);
}
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
// fp16 x fp16 -> fp32, M = 128; bit 16: B is MN-major.
__host__ __device__ constexpr uint32_t idesc(int n, bool b_mn) {
  return (1u << 4) | (uint32_t(b_mn) << 16) | (uint32_t(n >> 3) << 17) | (uint32_t(kTile >> 4) << 24);
}
template <uint32_t kAccumulate>
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t id) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 da, {%1, %4};\n\t"
      "mov.b64 db, {%2, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(id), "r"(kDescHigh), "n"(kAccumulate)
      : "memory");
}
template <uint32_t kAccumulate>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t id) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 db, {%2, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(id), "r"(kDescHigh), "n"(kAccumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t taddr, float* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
        "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]),
        "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]),
        "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {      // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// 64 rows of one head: `kAtoms` boxes of 64 values x 64 rows.
template <int D>
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int row) {
#pragma unroll
  for (int a = 0; a < Cfg<D>::kAtoms; ++a)
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst + a * Cfg<D>::kSliceBytes), "l"(map), "r"(bar), "r"(a * 64), "r"(head), "r"(row)
        : "memory");
}

// What a CTA works on: two tiles of `tokens` tokens each from token `first` on of one sequence.
struct Work {
  int q0, nq, k0, nk;        // the sequence's rows
  int first;
  __device__ __forceinline__ int limit(int token, int causal) const {   // keys that a token sees: 0 .. limit - 1
    const int most = causal ? min(nk, token + 1 + nk - nq) : nk;
    return max(most, 0);
  }
  // blocks of keys that some row of tile t sees
  __device__ __forceinline__ int blocks(int t, int tokens, int causal) const {
    const int a = first + t * tokens;
    if (a >= nq) return 0;
    return (limit(min(nq, a + tokens) - 1, causal) + kBlock - 1) / kBlock;
  }
};

struct Ends {
  int q0, q1, k0, k1;
};
__device__ __forceinline__ Ends sequence_ends(const Args& a, int b) {
  return {a.cu_q[b], a.cu_q[b + 1], a.cu_k[b], a.cu_k[b + 1]};
}
__device__ __forceinline__ int sequence_tiles(const Args& a, const Ends& e, Work* w) {
  w->q0 = e.q0;
  w->nq = e.q1 - e.q0;
  w->k0 = e.k0;
  w->nk = e.k1 - e.k0;
  if (w->nq <= 0) return 0;
  if (w->q0 < 0 || w->nq > a.total_q - w->q0 || w->k0 < 0 || w->nk < 0 || w->nk > a.total_k - w->k0) {
    atomicCAS(&g_prefill_status, 0, kRange);
    return 0;
  }
  return (w->nq + 2 * a.tokens - 1) / (2 * a.tokens);
}

// Ring entries of two blocks: K_0 and K_1 (which is always there, whatever it holds), then V_j and K_{j+2} for j = 0 .. n - 1
// (no keys with the last two).
template <int D>
struct Bars {
  static constexpr uint32_t kFull = Cfg<D>::kBarOffset, kEmpty = kFull + 8 * Cfg<D>::kStages, kS = kEmpty + 8 * Cfg<D>::kStages,
                            kP = kS + 32, kO = kP + 32, kQ = kO + 16, kGuard = kQ + 8, kGo = kGuard + 8 * kRaggedBlocks;
};

// The products of tile T, all issued by one thread, whose own instructions are part of the tile's pace: a wait or a commit takes it
// some 100 to 200 cycles, shared memory being busy with the operands.  So a ring entry holds what one step takes, values of this
// block and keys of the next but one, with one barrier.
template <int D, int T>
__device__ __forceinline__ void issue_products(uint32_t base, int n, int nt, int guarded, volatile int* abort_flag) {
  using C = Cfg<D>;
  using B = Bars<D>;
  constexpr uint32_t id_s = idesc(kBlock, false), id_o = idesc(D, true);
  constexpr uint32_t s_at = T * 128u, o_at = 256u + T * 128u;
  constexpr uint32_t ring = 2 * C::kTileBytes;
  const uint32_t q_desc = desc_k_major(base + T * C::kTileBytes);
  auto scores = [&](uint32_t buffer, uint32_t block_at) {             // S = Q K^T
    const uint32_t k = desc_k_major(block_at);
    mma_ss<0>(s_at + buffer * 64u, q_desc, k, id_s);
#pragma unroll
    for (int x = 1; x < D / 16; ++x)
      mma_ss<1>(s_at + buffer * 64u, q_desc + (x >> 2) * (C::kAtomBytes / 16) + (x & 3) * 2,
                k + (x >> 2) * (C::kSliceBytes / 16) + (x & 3) * 2, id_s);
    commit(base + B::kS + 8 * (2 * T + buffer));
  };
  if (!mbar_wait(base + B::kQ, 0, abort_flag, kSiteMma)) return;
  if (!mbar_wait(base + B::kFull, 0, abort_flag, kSiteMma)) return;
  fence_after();
  if (nt > 0) scores(0, base + ring);
  if (nt > 1) scores(1, base + ring + C::kBlockBytes);
  // no arrival is left under way when the CTA ends: only entries whose stage is filled again are released
  if (C::kStages <= n) commit(base + B::kEmpty);
  uint32_t stage = 1, phase = 0;
#pragma unroll 1
  for (int j = 0; j < n; ++j) {
    const uint32_t at = base + ring + stage * (2 * C::kBlockBytes), buffer = j & 1;
    if (!mbar_wait(base + B::kFull + 8 * stage, phase, abort_flag, kSiteMma)) return;
    if (j < nt) {
      if (j >= guarded && !mbar_wait(base + B::kGuard + 8 * (j - guarded), 0, abort_flag, kSiteMma)) return;
      if (!mbar_wait(base + B::kP + 8 * (2 * T + buffer), (j >> 1) & 1, abort_flag, kSiteMma)) return;
      fence_after();
      const uint32_t v = desc_mn_major(at);
      if (j == 0) mma_ts<0>(o_at, s_at + buffer * 64u, v, id_o);
      else mma_ts<1>(o_at, s_at + buffer * 64u, v, id_o);
#pragma unroll
      for (int x = 1; x < kBlock / 16; ++x) mma_ts<1>(o_at, s_at + buffer * 64u + 8u * x, v + 128 * x, id_o);
      if (j + 2 < nt) scores(buffer, at + C::kBlockBytes);
      else if (j + 1 < nt) commit(base + B::kS + 8 * (2 * T + buffer));       // says that this block's products are done
      else commit(base + B::kO + 8 * T);
    }
    if (j + 1 + C::kStages <= n) commit(base + B::kEmpty + 8 * stage);
    if (++stage == C::kStages) {
      stage = 0;
      phase ^= 1;
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
attn_prefill_kernel(const Args a, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                    const __grid_constant__ CUtensorMap v_map) {
  using C = Cfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];       // the kernel has no other shared memory
  const uint32_t base = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  // ---- barriers, tensor memory ----
  using B = Bars<D>;
  const uint32_t bar_full = base + B::kFull, bar_empty = base + B::kEmpty, bar_s = base + B::kS, bar_p = base + B::kP,
                 bar_o = base + B::kO, bar_q = base + B::kQ, bar_guard = base + B::kGuard, bar_go = base + B::kGo;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::kMiscOffset);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::kMiscOffset + 8);
  volatile int* not_finite = reinterpret_cast<volatile int*>(smem + C::kMiscOffset + 16);
  const unsigned long long wait_limit = warp == kLoadWarp ? g_prefill_wait_limit_ns : kWaitLimitNs;
  // a sequence per lane where a warp has enough of them: asked for before anything else
  Ends ends{0, 0, 0, 0};
  if (a.batch <= 32 && lane < a.batch) ends = sequence_ends(a, lane);
  if (tid == kThreads - 32) {
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(bar_full + 8 * i, 1);
      mbar_init(bar_empty + 8 * i, 2);
    }
    for (int i = 0; i < 4; ++i) {                   // tile i / 2, buffer i % 2
      mbar_init(bar_s + 8 * i, 1);
      mbar_init(bar_p + 8 * i, 4);
    }
    for (int t = 0; t < 2; ++t) mbar_init(bar_o + 8 * t, 1);
    mbar_init(bar_q, 1);
    for (int g = 0; g < kRaggedBlocks; ++g) {
      mbar_init(bar_guard + 8 * g, 1);
      mbar_init(bar_go + 8 * g, 1);
    }
    *abort_flag = 0;
    *not_finite = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kLoadWarp && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }

  // ---- which sequence and which of its tiles: the sequences' tile counts, added up by the whole CTA ----
  int* s_sums = reinterpret_cast<int*>(smem + C::kMiscOffset + 32);
  int& s_found = s_sums[kThreads / 32];
  int& s_local = s_sums[kThreads / 32 + 1];
  const int unit = int(blockIdx.x) % a.units;
  const int want = int(blockIdx.x) / a.units;
  if (tid == 0) s_found = -1;
  int found = -1, local = 0;
  Work w;
  if (a.batch <= 32) {                              // every warp for itself, a lane per sequence
    Work mine_w;
    const int mine = sequence_tiles(a, ends, &mine_w);
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    const uint32_t at = __ballot_sync(0xffffffffu, want < incl);
    found = at == 0 ? -1 : __ffs(at) - 1;
    const int owner = max(found, 0);
    local = __shfl_sync(0xffffffffu, incl, owner) - 1 - want;         // the longest rows of a sequence first
    w.q0 = __shfl_sync(0xffffffffu, mine_w.q0, owner);
    w.nq = __shfl_sync(0xffffffffu, mine_w.nq, owner);
    w.k0 = __shfl_sync(0xffffffffu, mine_w.k0, owner);
    w.nk = __shfl_sync(0xffffffffu, mine_w.nk, owner);
  } else {
    const int per = (a.batch + kThreads - 1) / kThreads;
    const int b0 = min(a.batch, tid * per), b1 = min(a.batch, b0 + per);
    int mine = 0;
    for (int b = b0; b < b1; ++b) mine += sequence_tiles(a, sequence_ends(a, b), &w);
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    if (lane == 31) s_sums[warp] = incl;
    __syncthreads();
    for (int i = 0; i < warp; ++i) incl += s_sums[i];
    int at = incl - mine;
    if (want >= at && want < incl) {
      for (int b = b0; b < b1; ++b) {
        const int n = sequence_tiles(a, sequence_ends(a, b), &w);
        if (want < at + n) {
          s_found = b;
          s_local = n - 1 - (want - at);            // the longest rows of a sequence first
          break;
        }
        at += n;
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (*tmem_slot != 0 && tid == 0) {
    *abort_flag = 1;
    atomicCAS(&g_prefill_status, 0, int(kSiteMma));
  }
  if (a.batch > 32) {
    found = s_found;
    local = s_local;
    if (found >= 0) sequence_tiles(a, sequence_ends(a, found), &w);
  }
  if (found < 0) {                                  // more CTAs than tiles: the grid is an upper bound
    if (warp == kMmaWarp)
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(*tmem_slot), "r"(512) : "memory");
    return;
  }
  w.first = local * 2 * a.tokens;
  const int kv = unit / a.chunks, chunk = unit % a.chunks;
  const int heads = min(a.heads_per_chunk, a.group - chunk * a.heads_per_chunk);
  const int head0 = kv * a.group + chunk * a.heads_per_chunk;
  const int n0 = w.blocks(0, a.tokens, a.causal), n1 = w.blocks(1, a.tokens, a.causal);
  const int n = max(n0, n1);
  // from this key on some row of the CTA does not see everything
  const int ragged = w.limit(w.first, a.causal);

  // All of tensor memory is this CTA's, so it starts at 0: addresses in it are constants.
  constexpr uint32_t tmem = 0;
  const uint32_t q_smem = base, ring = base + 2 * C::kTileBytes;

  if (warp < kSoftmaxWarps) {
    // ================= softmax of tile t: one thread per row =================
    const int t = warp >> 2;
    const int row = tid & 127;
    const int token = w.first + t * a.tokens + row / heads;
    const int head = head0 + row % heads;
    const bool live = row < a.tokens * heads && token < w.nq;
    const int limit = live ? w.limit(token, a.causal) : 0;
    const int nt = t == 0 ? n0 : n1;
    const uint32_t lanes = uint32_t(warp & 3) << 21;                 // tensor-memory lane 32 * (warp % 4)
    const uint32_t s_col = tmem + lanes + uint32_t(t) * 128u;
    const uint32_t o_col = tmem + lanes + 256u + uint32_t(t) * 128u;
    // first block of this tile with a key that some row does not see
    const int masked_from = w.limit(min(w.first + t * a.tokens, w.nq - 1), a.causal) / kBlock;
    float m = -INFINITY, l = 0.0f;
    float s[kBlock];
    bool ok = true;
    // The scores of block j into registers.  The copy is on its way when this returns.
    auto fetch = [&](int j) {
      if (!mbar_wait_warp(bar_s + 8 * (2 * t + (j & 1)), (j >> 1) & 1, abort_flag, kSiteSoftmax)) {
        ok = false;
        return;
      }
      fence_after();
      tmem_load32(s_col + 64 * (j & 1), s);
      tmem_load32(s_col + 64 * (j & 1) + 32, s + 32);
    };
    if (nt > 0) fetch(0);
    for (int j = 0; ok && j < nt; ++j) {
      tmem_wait_ld();
      if (a.sign != 1) {                                             // a scale that is not positive
#pragma unroll
        for (int i = 0; i < kBlock; ++i) s[i] *= float(a.sign);
      }
      if (j >= masked_from) {
        const int here = limit - j * kBlock;
#pragma unroll
        for (int i = 0; i < kBlock; ++i) s[i] = i < here ? s[i] : -INFINITY;
      }
      float top[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
      for (int i = 4; i < kBlock - 4; i += 8) {
#pragma unroll
        for (int x = 0; x < 4; ++x) top[x] = max_nan(top[x], s[i + x], s[i + 4 + x]);
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) top[x] = max_nan(top[x], s[kBlock - 4 + x]);
      float high = max_nan(max_nan(top[0], top[1], top[2]), top[3]) * a.c;
      if (high == INFINITY) high = NAN;                              // inf - inf
      const bool raise = limit > 0 && !(high <= m + kHeadroom);     // not for a row that is thrown away, whatever it holds
      if (j == 0) {
        m = high - kLead;
      } else if (__any_sync(0xffffffffu, raise)) {
        const float to = raise ? high - kLead : m;
        const float keep = to == -INFINITY ? 1.0f : exp2_fast(m - to);
        m = to;
        l *= keep;
        // O is at rest when the products of block j - 1 are done, which is what the next phase of that block's buffer says
        if (!mbar_wait_warp(bar_s + 8 * (2 * t + ((j - 1) & 1)), (((j - 1) >> 1) + 1) & 1, abort_flag, kSiteSoftmax)) {
          ok = false;
          break;
        }
        fence_after();
#pragma unroll 1
        for (int i = 0; i < D / 32; ++i) {
          float o[32];
          tmem_load32(o_col + 32 * i, o);
          tmem_wait_ld();
#pragma unroll
          for (int x = 0; x < 32; ++x) o[x] *= keep;
          tmem_store32(o_col + 32 * i, reinterpret_cast<const uint32_t*>(o));
        }
      }
      const float ref = m == -INFINITY ? 0.0f : m;
      const f32x2 c2 = pack2(a.c, a.c), r2 = pack2(-ref, -ref);
      f32x2 sum[2] = {pack2(0.0f, 0.0f), pack2(0.0f, 0.0f)};
      uint32_t p[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        float x, y;
        unpack2(fma2(pack2(s[2 * i], s[2 * i + 1]), c2, r2), x, y);
        x = exp2_fast(x);
        y = exp2_fast(y);
        sum[i & 1] = add2(sum[i & 1], pack2(x, y));
        p[i] = half2_bits(x, y);
      }
      tmem_store32(s_col + 64 * (j & 1), p);
      {
        float x, y;
        unpack2(add2(sum[0], sum[1]), x, y);
        l += x + y;
      }
      if (j + 1 < nt) fetch(j + 1);                                  // while the weights are on their way
      tmem_wait_st();
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_p + 8 * (2 * t + (j & 1)));
    }
    // ---- output ----
    if (ok && n > 0) {                               // a tile that sees no keys: its queries are still on their way
      ok = mbar_wait_warp(nt > 0 ? bar_o + 8 * t : bar_q, 0, abort_flag, kSiteOutput);
      fence_after();
    }
    if (ok) {
      const bool put_back = nt > 0 && *not_finite != 0;
      const float inv = limit > 0 ? 1.0f / l : 0.0f;
      __half* out = a.y + int64_t(w.q0 + token) * a.ldy + int64_t(head) * D;
      // Rows leave through the shared memory of the tile's queries, whose products are done, so that half a warp stores a row
      // at a time: a lane storing its own row would touch 32 lines an instruction.
      constexpr int kPieces = D / 8, kRowsAtOnce = 32 / kPieces;     // 16 bytes
      uint4* rows = reinterpret_cast<uint4*>(smem + t * C::kTileBytes) + (warp & 3) * 32 * kPieces;     // of this warp
      uint4* own = rows + lane * kPieces;
#pragma unroll 1
      for (int i = 0; i < D / 64; ++i) {
        float o[64];
        if (nt > 0) {
          tmem_load32(o_col + 64 * i, o);
          tmem_load32(o_col + 64 * i + 32, o + 32);
          tmem_wait_ld();
        }
#pragma unroll
        for (int x = 0; x < 64; ++x) o[x] = limit > 0 ? o[x] * inv : 0.0f;
        if (put_back) {
          for (int key = ragged; key < limit; ++key) {
            const __half* v = a.v + int64_t(w.k0 + key) * a.ldv + int64_t(kv) * D + 64 * i;
#pragma unroll
            for (int x = 0; x < 64; ++x) {
              const float f = __half2float(v[x]);
              if (!isfinite(f)) o[x] += f;
            }
          }
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          uint4 h;
          h.x = half2_bits(o[8 * x], o[8 * x + 1]);
          h.y = half2_bits(o[8 * x + 2], o[8 * x + 3]);
          h.z = half2_bits(o[8 * x + 4], o[8 * x + 5]);
          h.w = half2_bits(o[8 * x + 6], o[8 * x + 7]);
          own[(8 * i + x) ^ (lane & 7)] = h;
        }
      }
      __syncwarp();
      const uint64_t to = live ? reinterpret_cast<uint64_t>(out) : 0;
#pragma unroll 4
      for (int i = 0; i < 32 / kRowsAtOnce; ++i) {
        const int r = i * kRowsAtOnce + lane / kPieces, piece = lane % kPieces;
        uint4* at = reinterpret_cast<uint4*>(__shfl_sync(0xffffffffu, to, r));
        const uint4 h = rows[r * kPieces + (piece ^ (r & 7))];
        if (at != nullptr) at[piece] = h;
      }
    }
  } else if (warp < kLoadWarp) {
    // ================= products of tile t =================
    if (lane == 0 && n > 0) {
      if (warp == kMmaWarp) issue_products<D, 0>(base, n, n0, ragged / kBlock, abort_flag);
      else issue_products<D, 1>(base, n, n1, ragged / kBlock, abort_flag);
    }
  } else if (warp == kLoadWarp) {
    // ================= loads =================
    if (lane == 0 && n > 0 && wait_limit < kAtOnceNs) {
      *abort_flag = 1;
      atomicCAS(&g_prefill_status, 0, int(kSiteLoad));
    } else if (lane == 0 && n > 0) {
      // rows of a query tile: the chunk's heads of one token after another; what lies past the sequence is never stored
      mbar_expect(bar_q, (n1 > 0 ? 2 : 1) * C::kAtoms * 128 * a.heads_per_chunk * a.tokens);
      for (int t = 0; t < (n1 > 0 ? 2 : 1); ++t)
        for (int x = 0; x < C::kAtoms; ++x)
          asm volatile(
              "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
              ::"r"(q_smem + t * C::kTileBytes + x * C::kAtomBytes), "l"(&q_map), "r"(bar_q), "r"(x * 64), "r"(head0),
              "r"(w.q0 + w.first + t * a.tokens)
              : "memory");
      bool ok = true;
      for (int i = 0; ok && i <= n; ++i) {                            // ring entry i
        const int st = i % C::kStages;
        ok = i < C::kStages || mbar_wait(bar_empty + 8 * st, ((i / C::kStages) & 1) ^ 1, abort_flag, kSiteLoad);
        if (!ok) break;
        const uint32_t at = ring + uint32_t(st) * (2 * C::kBlockBytes);
        const bool keys = i == 0 || i + 1 < n;
        mbar_expect(bar_full + 8 * st, keys ? 2 * C::kBlockBytes : C::kBlockBytes);
        load_rows<D>(at, i == 0 ? &k_map : &v_map, bar_full + 8 * st, kv, w.k0 + (i == 0 ? 0 : i - 1) * kBlock);
        if (keys) load_rows<D>(at + C::kBlockBytes, &k_map, bar_full + 8 * st, kv, w.k0 + (i + 1) * kBlock);
        if (i - 1 >= ragged / kBlock) mbar_arrive(bar_go + 8 * (i - 1 - ragged / kBlock));
      }
    }
  } else {
    // ================= value rows that not all rows of the CTA see =================
    for (int j = ragged / kBlock; j < n; ++j) {
      const int g = j - ragged / kBlock;
      const int i = j + 1, s = i % C::kStages;
      // once the load is under way the entry's barrier is in this use's phase
      if (!mbar_wait_warp(bar_go + 8 * g, 0, abort_flag, kSiteGuard)) break;
      if (!mbar_wait_warp(bar_full + 8 * s, (i / C::kStages) & 1, abort_flag, kSiteGuard)) break;
      uint8_t* v = smem + 2 * C::kTileBytes + s * 2 * C::kBlockBytes;
      const int from = max(0, ragged - j * kBlock), end = w.nk - j * kBlock;     // rows to look at; rows past the sequence
      bool bad = false;
#pragma unroll 4
      for (int x = tid - 32 * kGuardWarp; x < (kBlock - from) * (D / 8); x += kGuardThreads) {
        const int r = from + x / (D / 8), piece = x % (D / 8);
        uint4* at = reinterpret_cast<uint4*>(v + (piece >> 3) * C::kSliceBytes + r * 128 + (piece & 7) * 16);
        if (r >= end) {
          *at = make_uint4(0, 0, 0, 0);
        } else {
          uint4 h = *at;
          uint32_t* u = reinterpret_cast<uint32_t*>(&h);
          bool found = false;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if ((u[k] & 0x7C00u) == 0x7C00u) { u[k] &= 0xFFFF0000u; found = true; }
            if ((u[k] & 0x7C000000u) == 0x7C000000u) { u[k] &= 0x0000FFFFu; found = true; }
          }
          if (found) *at = h;
          bad |= found;
        }
      }
      if (bad) *not_finite = 1;
      __threadfence_block();
      fence_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_guard + 8 * g);
    }
  }

  // ---- wind down ----
  __syncwarp();
  if (*abort_flag != 0) {                           // copies and products under way have time to land
    const unsigned long long t0 = now_ns();
    while (now_ns() - t0 < kDrainNs) __nanosleep(1000);
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// Test probe: a warp waits, through the kernel's own bounded waits, on a barrier that nobody arrives on.
__global__ void wait_expiry_kernel(int site) {
  __shared__ __align__(8) unsigned long long bar_storage;
  __shared__ int abort_word;
  const uint32_t bar = smem_u32(&bar_storage);
  if (threadIdx.x == 0) {
    abort_word = 0;
    mbar_init(bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  if (site != kSiteLoad && site != kSiteMma) (void)mbar_wait_warp(bar, 0, &abort_word, site);
  else if (threadIdx.x == 0) (void)mbar_wait(bar, 0, &abort_word, site);
}

// fp16 rows of `heads` heads of `dim` values: 64 values of `box_heads` heads of `box_rows` rows are copied at a time.
static bool row_map(CUtensorMap* map, const void* p, int64_t heads, int64_t dim, int64_t rows, int64_t ld, int box_heads,
                    int box_rows) {
  TensorMapEncodeFn encode = tensor_map_encoder();
  if (encode == nullptr) return false;
  const cuuint64_t dims[3] = {cuuint64_t(dim), cuuint64_t(heads), cuuint64_t(rows)};
  const cuuint64_t strides[2] = {cuuint64_t(dim) * 2, cuuint64_t(ld) * 2};
  const cuuint32_t box[3] = {64, cuuint32_t(box_heads), cuuint32_t(box_rows)}, steps[3] = {1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(p), dims, strides, box, steps,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
static int launch(const Args& a, const CUtensorMap& qm, const CUtensorMap& km, const CUtensorMap& vm, int64_t grid, cudaStream_t st) {
  if (!allow_dynamic_smem(reinterpret_cast<const void*>(&attn_prefill_kernel<D>), Cfg<D>::kSmemBytes)) return SMOOTHROT_CUDA_ERROR;
  attn_prefill_kernel<D><<<unsigned(grid), kThreads, Cfg<D>::kSmemBytes, st>>>(a, qm, km, vm);
  count_launch();
  return launch_status();
}

}  // namespace prefill
}  // namespace smoothrot

extern "C" {

int smoothrot_prefill_status_word(int* out, int clear) {
  if (cudaMemcpyFromSymbol(out, smoothrot::prefill::g_prefill_status, sizeof(int)) != cudaSuccess) return SMOOTHROT_CUDA_ERROR;
  if (clear && *out != 0) {
    const int zero = 0;
    if (cudaMemcpyToSymbol(smoothrot::prefill::g_prefill_status, &zero, sizeof(int)) != cudaSuccess) return SMOOTHROT_CUDA_ERROR;
  }
  return SMOOTHROT_OK;
}

int smoothrot_prefill_set_wait_limit_ns(uint64_t ns) {
  const unsigned long long v = ns == 0 ? smoothrot::prefill::kWaitLimitNs : static_cast<unsigned long long>(ns);
  return cudaMemcpyToSymbol(smoothrot::prefill::g_prefill_wait_limit_ns, &v, sizeof(v)) == cudaSuccess ? SMOOTHROT_OK
                                                                                                      : SMOOTHROT_CUDA_ERROR;
}

int smoothrot_prefill_wait_expiry(int site, void* stream) {
  smoothrot::prefill::wait_expiry_kernel<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>(site);
  smoothrot::count_launch();
  return smoothrot::launch_status();
}

int smoothrot_attn_prefill(const void* Q_f16, int64_t ldq, int64_t total_q, const void* K_f16, int64_t ldk, const void* V_f16,
                           int64_t ldv, int64_t total_k, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                           const int32_t* cu_q, const int32_t* cu_k, int64_t B, int causal, float scale, void* Y_f16,
                           int64_t ldy, void* stream) {
  using namespace smoothrot;
  using namespace smoothrot::prefill;
  // row and tile numbers stay well inside 32 bits
  const int64_t most = int64_t(1) << 30;
  if (total_q < 0 || total_k < 0 || total_q > most || total_k > most || B < 0 || B > 65535) return SMOOTHROT_INVALID_ARG;
  if (n_heads <= 0 || n_kv_heads <= 0 || n_heads > 65535 || n_heads % n_kv_heads != 0) return SMOOTHROT_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return SMOOTHROT_UNSUPPORTED_K;
  if ((causal & ~1) != 0 || !(scale == scale)) return SMOOTHROT_INVALID_ARG;
  if (total_q == 0 || B == 0) return SMOOTHROT_OK;
  const int64_t cq = n_heads * head_dim, ckv = n_kv_heads * head_dim;
  if (Q_f16 == nullptr || Y_f16 == nullptr || cu_q == nullptr || cu_k == nullptr || ldq < cq || ldy < cq) return SMOOTHROT_INVALID_ARG;
  if (total_k > 0 && (K_f16 == nullptr || V_f16 == nullptr || ldk < ckv || ldv < ckv)) return SMOOTHROT_INVALID_ARG;
  if (!aligned16(Q_f16) || !aligned16(Y_f16) || ldq % 8 != 0 || ldy % 8 != 0) return SMOOTHROT_BAD_ALIGNMENT;
  if (total_k > 0 && (!aligned16(K_f16) || !aligned16(V_f16) || ldk % 8 != 0 || ldv % 8 != 0)) return SMOOTHROT_BAD_ALIGNMENT;
  Args a;
  a.v = static_cast<const __half*>(V_f16);
  a.ldv = ldv; a.ldy = ldy;
  a.y = static_cast<__half*>(Y_f16);
  a.total_q = total_q; a.total_k = total_k;
  a.cu_q = cu_q; a.cu_k = cu_k;
  a.batch = int(B); a.causal = causal;
  a.group = int(n_heads / n_kv_heads);
  a.heads_per_chunk = a.group < kTile ? a.group : kTile;
  a.chunks = (a.group + kTile - 1) / kTile;
  a.tokens = kTile / a.heads_per_chunk;
  a.units = int(n_kv_heads) * a.chunks;
  a.sign = scale > 0.0f ? 1 : (scale < 0.0f ? -1 : 0);
  a.c = scale == 0.0f ? 1.0f : (scale < 0.0f ? -scale : scale) * 1.4426950408889634f;
  const int64_t grid = (total_q / (2 * a.tokens) + B) * a.units;
  if (grid > INT32_MAX) return SMOOTHROT_INVALID_ARG;
  CUtensorMap qm, km, vm;
  if (!row_map(&qm, Q_f16, n_heads, head_dim, total_q, ldq, a.heads_per_chunk, a.tokens)) return SMOOTHROT_CUDA_ERROR;
  km = vm = qm;                                     // the kernel prefetches all three
  if (total_k > 0) {
    if (!row_map(&km, K_f16, n_kv_heads, head_dim, total_k, ldk, 1, kBlock) ||
        !row_map(&vm, V_f16, n_kv_heads, head_dim, total_k, ldv, 1, kBlock))
      return SMOOTHROT_CUDA_ERROR;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return head_dim == 128 ? launch<128>(a, qm, km, vm, grid, st) : launch<64>(a, qm, km, vm, grid, st);
}

}  // extern "C"
