// Products of microscaled 4-bit floating point on tcgen05, which multiplies e2m1 codes and applies the groups' scales
// itself: the linear layer  Y = fp16(step_x[m] step_w[n] sum_g s_x s_w sum_{k in g} x w)  and the gated pair of
// projections  h = SiLU(gate) * up  with the next layer's encoding behind it.
//
// Nothing is widened or rearranged on the way: TMA brings packed codes (128 bytes = 256 codes a row and k-block,
// 128-byte swizzle) and whole blocks of scales into shared memory, tcgen05.cp copies the scales to tensor memory,
// tcgen05.mma reads both.  Two kernels:
//
//   pair    many tokens.  A cluster of two CTAs on a 256 x 256 tile (cta_group::2), persistent.
//   stream  few tokens.  The weights on the 128-row axis, the tokens on the other, K split over a cluster whose
//           partial sums meet in shared memory: bound by the one pass over the weights.
//
// Every wait on an mbarrier is bounded in wall time, as in the other kernels of the library.
#include <cuda.h>

#include <initializer_list>

#include "mx.cuh"

// defined with the norms: their timeout word and the limit of their waits
extern "C" int smoothrot_norm_status_word(int* out, int clear);
extern "C" int smoothrot_norm_set_wait_limit_ns(uint64_t ns);

namespace smoothrot {
namespace mx {

__device__ int g_mx_status = 0;
__device__ unsigned long long g_mx_wait_limit_ns = kWaitLimitNs;

enum Site { kPairLoad = 42, kPairAcc = 43, kPairFull = 44, kPairEpilogue = 45, kStreamLoad = 46, kStreamFull = 47,
            kStreamMixed = 48, kStreamEpilogue = 49, kProbe = 50 };

namespace {

constexpr int kTile = 128;            // rows of an operand in one CTA's shared memory
constexpr int kRowBytes = 128;        // of a k-block
constexpr int kBlockK = 256;          // codes of a k-block
constexpr int kStepsPerBlock = 4;     // an instruction takes 64 codes
constexpr int kTileBytes = kTile * kRowBytes;

// ---- PTX ----

// arrival on a barrier of this CTA or another of the cluster
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Waits for a phase; false if the limit has passed or another role of the CTA gave up.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int site) {
  if (bar_try(bar, parity)) return true;
  const unsigned long long t0 = now_ns();
  for (uint32_t spin = 1;; ++spin) {
    if (bar_try(bar, parity)) return true;
    if ((spin & 63u) == 0u) {
      if (*abort_flag != 0) return false;
      if (now_ns() - t0 > g_mx_wait_limit_ns) {
        *abort_flag = 1;
        atomicCAS(&g_mx_status, 0, site);
        return false;
      }
    }
  }
}
// The same for a whole warp, with one answer for all of its lanes.
__device__ __forceinline__ bool bar_wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag, int site) {
  return __all_sync(0xffffffffu, bar_wait(bar, parity, abort_flag, site));
}
// After a timeout copies and products that this CTA started may still be on their way: they land in microseconds.
__device__ __forceinline__ void drain_after_abort(volatile int* abort_flag) {
  if (*abort_flag != 0) drain();
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t map_to_cta(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
// into L2 alone, where what is written later still counts
__device__ __forceinline__ void tma_prefetch(const CUtensorMap* map, int x, int y) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}
// a load with a barrier that may be the other CTA's of the pair
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap* map, uint32_t src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
               ::"l"(map), "r"(src), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory"); }

// Matrix descriptors: only the low word, the address in 16 bytes, differs from one to the next.
// K-major operand, 128-byte swizzle: rows of 128 bytes, groups of 8 rows 1024 bytes apart.
constexpr uint32_t kCodesHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
// A block of scales: 32 rows of 16 bytes, no swizzle, groups of 8 rows 128 bytes apart.
constexpr uint32_t kScalesHigh = (128u >> 4) | (1u << 14);
__device__ __forceinline__ uint32_t desc_low(uint32_t addr) { return ((addr & 0x3FFFFu) >> 4) | (1u << 16); }
// Instruction descriptor: e2m1 x e2m1 -> fp32, K-major; which of a word's bytes are the scales of this
// step: bits 4-5 (B) and 29-30 (A); bit 23: scales are powers of two.
template <int GROUP>
__host__ __device__ constexpr uint32_t instruction(int m, int n, uint32_t scale_byte) {
  return (1u << 7) | (1u << 10) | (uint32_t(n >> 3) << 17) | (uint32_t(GROUP == 32) << 23) | (uint32_t(m >> 4) << 24) |
         (scale_byte << 4) | (scale_byte << 29);
}
// These are issued by one thread at one a few dozen clocks, against 128 clocks that the tensor core takes for the largest: a
// warp that is known to be of one mind, one elected lane and 32-bit operands keep the issue short (67 clocks a product with a
// lane that was told apart by its number and whole 64-bit descriptors, 39 so).
template <int GROUP, int CTAS>
__device__ __forceinline__ void mma(uint32_t d, uint32_t a, uint32_t b, uint32_t inst, uint32_t scale_a, uint32_t scale_b,
                                    uint32_t accumulate) {
#define SR_MX_MMA(CG, KIND)                                                                                       \
  asm volatile(                                                                                                   \
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"                                                             \
      "setp.ne.b32 p, %6, 0;\n\t"                                                                                 \
      "mov.b64 da, {%1, %7};\n\t"                                                                                 \
      "mov.b64 db, {%2, %7};\n\t"                                                                                 \
      "tcgen05.mma.cta_group::" CG "." KIND " [%0], da, db, %3, [%4], [%5], p;\n\t}" ::"r"(d),                    \
      "r"(a), "r"(b), "r"(inst), "r"(scale_a), "r"(scale_b), "r"(accumulate), "r"(kCodesHigh)                     \
      : "memory")
  if constexpr (GROUP == 32 && CTAS == 2) SR_MX_MMA("2", "kind::mxf4.block_scale.scale_vec::2X");
  if constexpr (GROUP == 32 && CTAS == 1) SR_MX_MMA("1", "kind::mxf4.block_scale.scale_vec::2X");
  if constexpr (GROUP == 16 && CTAS == 2) SR_MX_MMA("2", "kind::mxf4nvf4.block_scale.scale_vec::4X");
  if constexpr (GROUP == 16 && CTAS == 1) SR_MX_MMA("1", "kind::mxf4nvf4.block_scale.scale_vec::4X");
#undef SR_MX_MMA
}
// 512 bytes of scales to 4 columns of tensor memory
template <int CTAS>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t desc) {
  if constexpr (CTAS == 2)
    asm volatile("{\n\t.reg .b64 d;\n\tmov.b64 d, {%1, %2};\n\ttcgen05.cp.cta_group::2.32x128b.warpx4 [%0], d;\n\t}"
                 ::"r"(tmem), "r"(desc), "r"(kScalesHigh) : "memory");
  else
    asm volatile("{\n\t.reg .b64 d;\n\tmov.b64 d, {%1, %2};\n\ttcgen05.cp.cta_group::1.32x128b.warpx4 [%0], d;\n\t}"
                 ::"r"(tmem), "r"(desc), "r"(kScalesHigh) : "memory");
}
__device__ __forceinline__ bool elected() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
// The warp's number, as a value that is the same in all its lanes.
__device__ __forceinline__ int warp_number() { return __shfl_sync(0xffffffffu, int(threadIdx.x >> 5), 0); }
// A place in a ring of N stages and the parity of the phase that it is in.
template <int N>
struct Ring {
  int s = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next() {
    if (++s == N) {
      s = 0;
      phase ^= 1u;
    }
  }
};
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void commit_pair(uint32_t bar) {
  const uint16_t both = 3;
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(bar), "h"(both) : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t cols) {
  if constexpr (CTAS == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
}
template <int CTAS>
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t cols) {
  if constexpr (CTAS == 2)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
  else
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t taddr, float (&v)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load(uint32_t taddr, float (&v)[8]) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---- what the epilogues share ----

// g / (1 + 2^(-g log2 e)) * u, two at a time; a power beyond the range gives 0 or g.  The power's argument is rounded to fp32 and the
// reciprocal is the hardware's, so the result is off by some |g| units in the last place: in front of a rounding to fp16 alone, which hides
// it.  Numerator and denominator are quartered, so that the reciprocal of the largest finite sum is a normal number.
__device__ __forceinline__ f32x2 silu_times(f32x2 g, f32x2 u) {
  const f32x2 quarter = pack2(0.25f, 0.25f);
  const float minus = -1.44269504f;      // log2 e
  float t[2], e[2], r[2];
  unpack2(mul2(g, pack2(minus, minus)), t[0], t[1]);
#pragma unroll
  for (int i = 0; i < 2; ++i) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e[i]) : "f"(t[i]));
  unpack2(fma2(pack2(e[0], e[1]), quarter, quarter), t[0], t[1]);
#pragma unroll
  for (int i = 0; i < 2; ++i) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r[i]) : "f"(t[i]));
  return mul2(mul2(mul2(g, quarter), pack2(r[0], r[1])), u);
}
// The same in front of codes, whose borders show the last bit: the library's exponential, and a quotient with one residual correction,
// as the gated product of the integer layers has them.  Of 1.4e9 values of blocks of 14336 features none was coded otherwise than with an
// IEEE division, which leaves its fast path at zeros (those of rows past the last: 300 x 5632 x 2048 in groups of 16 22 us, this 12.5, the
// form above 11.2, where 128 of those values got another code).  Where the power is infinite the reciprocal is 0, and where g is
// infinite the residual is no number: either way the correction is held to what changes nothing.
__device__ __forceinline__ f32x2 silu_exact(f32x2 g, f32x2 u) {
  const f32x2 quarter = pack2(0.25f, 0.25f), minus = pack2(-0.25f, -0.25f);
  float e[2], s[2], r[2], d[2];
  unpack2(g, e[0], e[1]);
#pragma unroll
  for (int i = 0; i < 2; ++i) e[i] = expf(-e[i]);
  const f32x2 sum = fma2(pack2(e[0], e[1]), minus, minus);      // -(1 + e) / 4
  unpack2(sum, s[0], s[1]);
#pragma unroll
  for (int i = 0; i < 2; ++i) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r[i]) : "f"(-s[i]));
  const f32x2 inv = pack2(r[0], r[1]), part = mul2(g, quarter), q = mul2(part, inv);
  unpack2(fma2(sum, q, part), d[0], d[1]);
  return mul2(fma2(pack2(fmaxf(d[0], -1e36f), fmaxf(d[1], -1e36f)), inv, q), u);
}

// A thread's 32 neighbouring values to codes; the scale bytes of their one or two groups in the low bits of the result.
template <int GROUP>
__device__ __forceinline__ uint32_t encode_values(const f32x2 (&v)[16], float step, uint4* codes) {
  const RowStep row = GROUP == 16 ? row_step(step) : RowStep{};
  uint32_t bytes = 0;
  uint32_t* out = reinterpret_cast<uint32_t*>(codes);
#pragma unroll
  for (int g = 0; g < 32 / GROUP; ++g) {
    constexpr int W = GROUP / 2;
    f32x2 part[W];
#pragma unroll
    for (int i = 0; i < W; ++i) part[i] = v[g * W + i];
    uint32_t byte;
    const Part<W / 4> c = encode<GROUP, true>(part, top_of(part), row, &byte);
    bytes |= byte << (8 * g);
#pragma unroll
    for (int i = 0; i < W / 4; ++i) out[g * (W / 4) + i] = c.w[i];
  }
  return bytes;
}

// 32 columns of a row times its step and the columns', which lie at `at` in shared memory (0: none).
__device__ __forceinline__ void times_steps(f32x2 (&v)[16], float row, uint32_t at) {
  const f32x2 row2 = pack2(row, row);
  if (at == 0u) {
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = mul2(v[j], row2);
    return;
  }
#pragma unroll
  for (int j = 0; j < 16; j += 2) {
    float4 w;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(w.x), "=f"(w.y), "=f"(w.z), "=f"(w.w) : "r"(at + 8u * j) : "memory");
    v[j] = mul2(v[j], mul2(row2, pack2(w.x, w.y)));
    v[j + 1] = mul2(v[j + 1], mul2(row2, pack2(w.z, w.w)));
  }
}

// A warp's 32 rows x 32 columns to fp16 through its box in shared memory (64-byte swizzle) and TMA, which clips at the matrix's
// edges: rows of 64 bytes leave whole.
__device__ __forceinline__ void store_box(const CUtensorMap* map, uint32_t box, const f32x2 (&v)[16], int x, int y, int n, int m,
                                          int lane) {
  if (lane == 0) store_wait_read<0>();
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x2 part[4] = {v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
    const Part<4> h = narrow(part);
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                 ::"r"(box + uint32_t(lane) * 64u + ((uint32_t(j) ^ uint32_t((lane >> 1) & 3)) << 4)), "r"(h.w[0]), "r"(h.w[1]),
                   "r"(h.w[2]), "r"(h.w[3]) : "memory");
  }
  fence_async();
  __syncwarp();
  if (lane == 0) {
    if (x < n && y < m) tma_store(map, box, x, y);
    store_commit();
  }
}

enum Mode { kLinear = 0, kGatedHalf = 1, kGatedCodes = 2 };

struct Args {
  int M, N;                   // tokens, output channels (of one projection)
  int kblocks, last_steps;    // k-blocks, instructions of the last one
  int tiles_a, tiles_b;
  const float *x_step, *w_step, *up_step;   // per row, or null
  __half* y;
  int64_t ldy;
  uint8_t *q_out, *scale_out;
  const float* h_step;
  int walsh;
  float norm;
};

// ---------------------------------------------------------------------------
// Many tokens: 256 x 256 tiles over a pair of CTAs.
//
// Each CTA stages 128 token rows and half of the 256 weight rows (gated: one CTA the gate's 128 rows, the other the
// up projection's), the pair's tensor cores share the halves.  Scales of the weights are applied column by
// column in both CTAs, so each holds all of them.  A 4-bit operand row of an instruction is 32 bytes like any other
// type's, so the pair moves 16 KB through shared memory per CTA and 128-clock instruction: the layout with the least.
//
// Tensor memory: two accumulators of 256 columns and the scales of a k-block (24 or 48 columns) are more than 512, so the
// second accumulator starts 224 (208) columns after the first and they share 32 (48).  The epilogue's warps take a whole accumulator
// into registers at once, and the next tile's products wait only for those that hold shared columns.
//
// Warps: 0 TMA, 1 products (of the first CTA), 2..17 epilogue, four to a quadrant of tensor-memory lanes, a chunk of columns
// each: with two to a quadrant a gated tile's activation and encoding took longer than its products.
//
// 2048 x 4096 x 14336: 42 us (5.7 PFLOP/s) to 60 once the power cap bites; 8192 x 4096 x 14336 168 to 173 (5.6 to 5.7), with codes of
// zeros 132 (7.3 of 9.2 that 128 clocks a product allow; the way from L2, 56 bytes a clock and SM, is next); 700 x 4096 x 4096 9.8, of which 4.6
// are the start and the end.
// ---------------------------------------------------------------------------
template <int GROUP>
struct Pair {
  static constexpr int kAtoms = kBlockK / GROUP / kAtomGroups;      // blocks of scales per 128 rows and k-block
  static constexpr int kScaleBytes = kAtoms * kAtomBytes;
  static constexpr int kStageBytes = 2 * kTileBytes + 3 * kScaleBytes;
  static constexpr int kStages = 5;
  static constexpr int kEpiWarps = 16, kThreads = 32 * (2 + kEpiWarps);
  static constexpr int kBoxBytes = 32 * 64;                         // 32 rows x 32 fp16
  static constexpr int kOutBytes = kEpiWarps * kBoxBytes;
  static constexpr int kBarriers = 2 * kStages + 5;
  static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kOutBytes + kBarriers * 8 + 16;
  static constexpr int kSecond = GROUP == 32 ? 224 : 208;           // first column of the second accumulator
  static constexpr int kScaleCol = kSecond + 256;                   // scales of A, then of B
  static_assert(kScaleCol + 12 * kAtoms <= 512, "tensor memory");
  static_assert(kSmemBytes <= 227 * 1024, "shared memory");
  static_assert(kStageBytes % 1024 == 0, "swizzled tiles start on 1024 bytes");
};

// A k-block's scale copies and products; `sc` is the block's scales (A, then the two halves of B), all as low words.
template <int GROUP, int STEPS>
__device__ __forceinline__ void pair_block(uint32_t acc, uint32_t a, uint32_t b, uint32_t sc, uint32_t sa, uint32_t sb, bool fresh) {
  using T = Pair<GROUP>;
  constexpr int per = kStepsPerBlock / T::kAtoms;      // products that an atom of scales serves
#pragma unroll
  for (int j = 0; j < STEPS; ++j) {
    const int atom = j / per;
    if (j % per == 0) {
      copy_scales<2>(sa + 4 * atom, sc + atom * (kAtomBytes / 16));
      copy_scales<2>(sb + 8 * atom, sc + (T::kScaleBytes + atom * kAtomBytes) / 16);
      copy_scales<2>(sb + 8 * atom + 4, sc + (2 * T::kScaleBytes + atom * kAtomBytes) / 16);
    }
    mma<GROUP, 2>(acc, a + 2 * j, b + 2 * j, instruction<GROUP>(256, 256, GROUP == 32 ? 2 * (j % 2) : 0), sa + 4 * atom,
                  sb + 8 * atom, j > 0 || !fresh);
  }
}

template <int GROUP, int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Pair<GROUP>::kThreads, 1)
mx_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ CUtensorMap map_u, const __grid_constant__ CUtensorMap map_sa,
               const __grid_constant__ CUtensorMap map_sb, const __grid_constant__ CUtensorMap map_su,
               const __grid_constant__ CUtensorMap map_y, const Args p) {
  using T = Pair<GROUP>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t base = (raw_addr + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (base - raw_addr);
  const uint32_t out_base = base + T::kStages * T::kStageBytes;
  const uint32_t bar_base = out_base + T::kOutBytes;
  auto full = [&](int s) { return bar_base + 8u * s; };                       // in the first CTA, for both
  auto empty = [&](int s) { return bar_base + 8u * (T::kStages + s); };       // in each
  const uint32_t acc_full = bar_base + 8u * (2 * T::kStages);                 // one per accumulator, in each
  const uint32_t acc_empty = acc_full + 16u;                                  // one per accumulator, in the first CTA
  const uint32_t acc_shared = acc_empty + 16u;                                // the columns that both hold, in the first CTA
  constexpr int kHolders = MODE != kLinear && GROUP == 16 ? 2 : 1;            // chunks with shared columns
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + (bar_base - base) + 8 * T::kBarriers);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = warp_number(), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  // Set-up: barriers, which both CTAs have to have before a load of either is issued, and tensor memory meanwhile.
  if (warp == 0) {
    if (elected()) {
      for (int s = 0; s < T::kStages; ++s) {
        bar_init(full(s), 1);
        bar_init(empty(s), 1);
      }
      bar_init(acc_full, 1);
      bar_init(acc_full + 8u, 1);
      bar_init(acc_empty, 2 * T::kEpiWarps);
      bar_init(acc_empty + 8u, 2 * T::kEpiWarps);
      bar_init(acc_shared, 2 * 4 * kHolders);
      *abort_flag = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      fence_async();
    }
    __syncwarp();
  }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  if (warp == 1) tmem_alloc<2>(smem_u32(tmem_slot), 512);
  if (warp == 2 && elected()) {
    // While the call before finishes, this CTA's first weights are asked into L2: 2 % of calls with 200 to 1500 tokens.  Whatever was asked
    // for after the wait, ahead of the ring, cost more than it gave (4 % in the mean).
    const int tb = int(blockIdx.x >> 1) / p.tiles_a;
    const bool up = MODE != kLinear && rank == 1;
    const int row = MODE != kLinear ? tb : 2 * tb + int(rank);
    for (int kb = 0; kb < min(p.kblocks, 2); ++kb) {
      tma_prefetch(up ? &map_u : &map_b, kb * kRowBytes, row * kTile);
      tma_prefetch(up ? &map_su : &map_sb, kb * (T::kScaleBytes / 8), row);
    }
  }
  __syncwarp();
  after_the_call_before();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (warp != 0) {
    fence_before();
    asm volatile("bar.sync 1, %0;" ::"n"(T::kThreads - 32) : "memory");
    fence_after();
  }
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);       // in warp 0, which has no use for it, anything
  const int tiles = p.tiles_a * p.tiles_b;
  const int first = blockIdx.x >> 1, step = gridDim.x >> 1;

  if (warp == 0) {
    const bool one = elected();
    const CUtensorMap* mb = MODE != kLinear && rank == 1 ? &map_u : &map_b;
    const CUtensorMap* ms1 = MODE != kLinear ? &map_su : &map_sb;
    if (one) {
      prefetch_map(&map_a);
      prefetch_map(mb);
      prefetch_map(&map_sa);
      prefetch_map(&map_sb);
      prefetch_map(ms1);
    }
    Ring<T::kStages> r;
    const uint32_t lead = map_to_cta(bar_base, 0);
    bool ok = true;
    for (int tile = first; tile < tiles && ok; tile += step) {
      const int ta = tile % p.tiles_a, tb = tile / p.tiles_a;
      const int row_a = ta * 256 + int(rank) * kTile;
      const int row_b = MODE != kLinear ? tb * kTile : tb * 256 + int(rank) * kTile;
      const int sb0 = MODE != kLinear ? tb : 2 * tb, sb1 = MODE != kLinear ? tb : 2 * tb + 1;
      for (int kb = 0; kb < p.kblocks; ++kb, r.next()) {
        ok = bar_wait_warp(empty(r.s), r.phase ^ 1u, abort_flag, kPairLoad);
        if (!ok) break;
        if (one) {
          if (rank == 0) bar_expect(full(r.s), 2u * T::kStageBytes);
          const uint32_t bar = lead + 8u * r.s;
          const uint32_t dst = base + r.s * T::kStageBytes, sc = dst + 2 * kTileBytes;
          tma_load_pair(dst, &map_a, bar, kb * kRowBytes, row_a);
          tma_load_pair(dst + kTileBytes, mb, bar, kb * kRowBytes, row_b);
          const int x = kb * (T::kScaleBytes / 8);
          tma_load_pair(sc, &map_sa, bar, x, row_a / kTile);
          tma_load_pair(sc + T::kScaleBytes, &map_sb, bar, x, sb0);
          tma_load_pair(sc + 2 * T::kScaleBytes, ms1, bar, x, sb1);
        }
        __syncwarp();
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const bool one = elected();
      const uint32_t sa = tmem + T::kScaleCol, sb = sa + 4 * T::kAtoms;
      Ring<T::kStages> r;
      uint32_t n = 0;
      bool ok = true;
      for (int tile = first; tile < tiles && ok; tile += step, ++n) {
        // the tile before the last has left this accumulator, and the last one the columns that it shares with it
        if (!bar_wait_warp(acc_empty + 8u * (n & 1u), ((n >> 1) & 1u) ^ 1u, abort_flag, kPairAcc)) break;
        if (!bar_wait_warp(acc_shared, (n & 1u) ^ 1u, abort_flag, kPairAcc)) break;
        fence_after();
        const uint32_t acc = tmem + ((n & 1u) ? T::kSecond : 0);
        for (int kb = 0; kb < p.kblocks; ++kb, r.next()) {
          ok = bar_wait_warp(full(r.s), r.phase, abort_flag, kPairFull);
          if (!ok) break;
          fence_after();
          if (one) {
            const uint32_t src = desc_low(base + r.s * T::kStageBytes);
            const uint32_t b = src + kTileBytes / 16, sc = src + 2 * kTileBytes / 16;
            if (kb + 1 < p.kblocks || p.last_steps == kStepsPerBlock)
              pair_block<GROUP, kStepsPerBlock>(acc, src, b, sc, sa, sb, kb == 0);
            else
              pair_block<GROUP, kStepsPerBlock / 2>(acc, src, b, sc, sa, sb, kb == 0);
            commit_pair(empty(r.s));
          }
          __syncwarp();
        }
        if (ok && one) commit_pair(acc_full + 8u * (n & 1u));
        __syncwarp();
      }
    }
  } else {
    const int q = warp & 3;                    // quadrant of tensor-memory lanes
    const uint32_t box = out_base + uint32_t(warp - 2) * T::kBoxBytes;
    const uint32_t acc_free = map_to_cta(acc_empty, 0), shared_free = map_to_cta(acc_shared, 0);
    const bool steps = p.x_step != nullptr || p.w_step != nullptr || p.up_step != nullptr || (MODE == kGatedCodes && GROUP == 16);
    const int chunk = (warp - 2) >> 2;
    // the tile's place and the next one's, without a division for each
    int ta = first % p.tiles_a, tb = first / p.tiles_a;
    const int step_a = step % p.tiles_a, step_b = step / p.tiles_a;
    // A tile's steps are asked for while the one before is finished, each lane those of its row and of a column of either part; the
    // columns' then go round through the warp's box (512 x 5632 x 2048 gated with all steps 12.8 us where each lane loaded all columns', of
    // which 2 were those loads).  In front of codes they are asked for behind the gate, which wants the registers (in groups of 16, 512 x
    // 5632 x 2048, 12.9 us -> 12.5).
    const float* second = MODE == kLinear ? p.w_step : p.up_step;
    const bool column_steps = p.w_step != nullptr || second != nullptr;
    float xs_next = 1.0f, hs_next = 1.0f, w_next = 1.0f, w2_next = 1.0f;
    auto row_of = [&] { return ta * 256 + int(rank) * kTile + q * 32; };
    auto column_of = [&] { return MODE == kLinear ? tb * 256 + 64 * chunk : tb * kTile + 32 * chunk; };
    auto ask = [&] {
      const int m = row_of() + lane, n = column_of() + lane, n2 = MODE == kLinear ? n + 32 : n;
      if (p.x_step != nullptr && m < p.M) xs_next = load(p.x_step + m);
      if (MODE == kGatedCodes && GROUP == 16 && m < p.M) hs_next = load(p.h_step + m);
      if (p.w_step != nullptr && n < p.N) w_next = load(p.w_step + n);
      if (second != nullptr && n2 < p.N) w2_next = load(second + n2);
    };
    if (first < tiles) ask();
    uint32_t n = 0;
    for (int tile = first; tile < tiles; tile += step, ++n) {
      const int row0 = row_of(), m = row0 + lane, n0 = column_of();
      const float xs = xs_next, hs = hs_next, w = w_next, w2 = w2_next;
      // where the chunk's two parts of 32 columns lie in the accumulator
      const int col_a = MODE == kLinear ? 64 * chunk : 32 * chunk, col_b = MODE == kLinear ? col_a + 32 : 128 + col_a;
      if (!bar_wait_warp(acc_full + 8u * (n & 1u), (n >> 1) & 1u, abort_flag, kPairEpilogue)) break;
      fence_after();
      const uint32_t acc = tmem + (uint32_t(q * 32) << 16) + ((n & 1u) ? T::kSecond : 0);
      uint32_t raw_a[32], raw_b[32];
      tmem_load32(acc + col_a, raw_a);
      tmem_load32(acc + col_b, raw_b);
      tmem_wait_ld();
      fence_before();
      __syncwarp();
      if (lane == 0) {
        // the shared columns are the last of the first accumulator and the first of the second
        if ((n & 1u) ? chunk < kHolders : chunk >= 4 - kHolders) bar_arrive_cluster(shared_free);
        bar_arrive_cluster(acc_free + 8u * (n & 1u));
      }
      ta += step_a;
      tb += step_b;
      if (ta >= p.tiles_a) {
        ta -= p.tiles_a;
        ++tb;
      }
      if (MODE != kGatedCodes && steps && tile + step < tiles) ask();
      f32x2 a[16], b[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        a[j] = pack2(__uint_as_float(raw_a[2 * j]), __uint_as_float(raw_a[2 * j + 1]));
        b[j] = pack2(__uint_as_float(raw_b[2 * j]), __uint_as_float(raw_b[2 * j + 1]));
      }
      if (steps) {
        if (column_steps) {
          if (MODE != kGatedCodes && lane == 0) store_wait_read<0>();
          __syncwarp();
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(box + 4u * lane), "f"(w) : "memory");
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(box + 128u + 4u * lane), "f"(w2) : "memory");
          __syncwarp();
        }
        times_steps(a, xs, column_steps ? box : 0u);
        times_steps(b, xs, column_steps ? box + 128u : 0u);
      }
      if constexpr (MODE == kLinear) {
        store_box(&map_y, box, a, n0, row0, p.N, p.M, lane);
        store_box(&map_y, box, b, n0 + 32, row0, p.N, p.M, lane);
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) a[j] = MODE == kGatedCodes ? silu_exact(a[j], b[j]) : silu_times(a[j], b[j]);
        if (MODE == kGatedCodes && steps && tile + step < tiles) ask();
        if (p.walsh) walsh_rows<32>(a, p.norm, lane);
        if constexpr (MODE == kGatedHalf) {
          store_box(&map_y, box, a, n0, row0, p.N, p.M, lane);
        } else {
          uint4 codes;
          const uint32_t bytes = encode_values<GROUP>(a, hs, &codes);
          if (m < p.M && n0 < p.N) {
            __stcs(reinterpret_cast<uint4*>(p.q_out + int64_t(m) * (p.N / 2) + n0 / 2), codes);
            uint8_t* to = p.scale_out + scale_word(m, n0 / (4 * GROUP), p.N / (4 * GROUP)) + (n0 / GROUP & 3);
            if constexpr (GROUP == 32) *to = uint8_t(bytes);
            else *reinterpret_cast<uint16_t*>(to) = uint16_t(bytes);
          }
        }
      }
    }
    if (MODE != kGatedCodes && lane == 0) store_wait_read<0>();      // the box may go; what was stored arrives before the grid ends
  }

  // a CTA that gave up tells the other, which waits for it before it leaves
  if (*abort_flag != 0)
    asm volatile("st.shared::cluster.u32 [%0], %1;"
                 ::"r"(map_to_cta(smem_u32(const_cast<const int*>(abort_flag)), rank ^ 1u)), "r"(1u) : "memory");
  drain_after_abort(abort_flag);
  fence_before();
  __syncthreads();
  cluster_sync();
  if (warp == 1) {
    __syncwarp();
    fence_after();
    tmem_free<2>(tmem, 512);
  }
}

// ---------------------------------------------------------------------------
// Few tokens: the weights on the 128-row axis, BN tokens on the other.
//
// The one pass over the weights is what such a call costs, so the kernel keeps as much of it in flight as shared memory holds:
// a ring of 16 KB weight tiles with their scales, and the tokens' BN rows beside them.  A gated tile is 64 rows of the gate and
// the 64 rows of the up projection beside it; a warp puts its block of scales together from the halves of the two that hold
// them (a copy to tensor memory starts at a multiple of 4 columns, so halves cannot be laid side by side there).  One CTA computes a tile over one part of K; the parts of a tile are a
// cluster, send each other the sums of the tokens that the other finishes, and each adds up its own over all parts, in the
// parts' order: the same bits from call to call.
//
// Where K is not split, two CTAs fit an SM, which evens out tiles that are not a multiple of the SMs, and lets a call's first loads be
// issued while the call before is finishing.  Where it is split, the places of the sums lie behind the ring and one CTA fits, two in
// three forms (16 tokens and groups of 32; gated: 32 tokens and groups of 32, 16 and groups of 16).
//
// Warps: 0 TMA, 1 products, 2..9 read the accumulator, two to a quadrant of its lanes, and finish; 2 mixes scales before.
//
// 1 x 4096 x 14336: 7.9 us (4.0 TB/s over all, 5.7 between the first byte and the last), gated 1 x 14336 x 4096 into codes 13.3 (4.7 TB/s),
// 61 x 4096 x 4096 5.0, 128 x 4096 x 14336 11.6; weights from memory.
// ---------------------------------------------------------------------------
constexpr int kStreamThreads = 320;

template <int GROUP, int BN, bool GATED>
struct Stream {
  static constexpr int kAtoms = kBlockK / GROUP / kAtomGroups;
  static constexpr int kScaleBytes = kAtoms * kAtomBytes;
  static constexpr int kTokenBytes = BN * kRowBytes;
  static constexpr int kScales = GATED ? 3 : 2;                  // weights' (gate's and up's), tokens'
  static constexpr int kStageBytes = kTileBytes + kTokenBytes + kScales * kScaleBytes;
  static constexpr int kStages = 110 * 1024 / kStageBytes;
  static constexpr int kTileRows = GATED ? kTile / 2 : kTile;    // output channels of a tile
  static constexpr int kBarriers = (GATED ? 3 : 2) * kStages + 1;
  static constexpr int kRingBytes = kStages * kStageBytes;
  // of one part: over the ring, once it has been used; of more: behind it, rounded up to whole rows of tokens (3 parts: BN + 2)
  static constexpr int kSumBytes = (BN + 2) * kTile * 4;
  static constexpr int kHeadBytes = (kBarriers * 8 + 16 + 127) / 128 * 128;
  static constexpr int kSmemBytes = 1024 + kRingBytes + kHeadBytes;
  static constexpr int kScaleCol = BN;
  static constexpr int kCols = kScaleCol + 8 * kAtoms;           // weights' scales, tokens' scales
  static constexpr int kTmemCols = kCols <= 32 ? 32 : kCols <= 64 ? 64 : kCols <= 128 ? 128 : 256;
  static_assert(kCols <= 256, "tensor memory of two CTAs");
  static_assert(kSumBytes <= kRingBytes && 2 * (kSmemBytes + 1024) <= 228 * 1024, "shared memory of two CTAs of one part");
  static_assert(kSmemBytes + kSumBytes <= 227 * 1024, "shared memory of a CTA of more parts");
  static_assert(kStageBytes % 1024 == 0, "swizzled tiles start on 1024 bytes");
};

// Eight neighbouring sums of a part; every other four lanes take the halves in the other order, and no two meet in a bank.
__device__ __forceinline__ void add_shared(float (&v)[8], uint32_t addr) {
  const bool other = (threadIdx.x & 4) != 0;
  const uint32_t flip = other ? 16u : 0u;
  float4 a, b;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(a.x), "=f"(a.y), "=f"(a.z), "=f"(a.w) : "r"(addr + flip) : "memory");
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(b.x), "=f"(b.y), "=f"(b.z), "=f"(b.w) : "r"(addr + (16u - flip)) : "memory");
  v[0] += other ? b.x : a.x; v[1] += other ? b.y : a.y; v[2] += other ? b.z : a.z; v[3] += other ? b.w : a.w;
  v[4] += other ? a.x : b.x; v[5] += other ? a.y : b.y; v[6] += other ? a.z : b.z; v[7] += other ? a.w : b.w;
}
__device__ __forceinline__ void eight_steps(const float* step, int n, float (&w)[8]) {
  float4 a = make_float4(1.0f, 1.0f, 1.0f, 1.0f), b = a;
  if (step != nullptr) {
    a = load(reinterpret_cast<const float4*>(step + n));
    b = load(reinterpret_cast<const float4*>(step + n) + 1);
  }
  w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
  w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
}

// A k-block's scale copies and products; `src` is the stage's low word, `sa` the first column of scales.  All copies
// come first: 1.3 % faster over 56 sizes than each in front of the products that need it.
template <int GROUP, int BN, bool GATED, int STEPS>
__device__ __forceinline__ void stream_block(uint32_t acc, uint32_t src, uint32_t sa, bool fresh) {
  using T = Stream<GROUP, BN, GATED>;
  constexpr int per = kStepsPerBlock / T::kAtoms;
  const uint32_t tokens = src + kTileBytes / 16, sc = tokens + T::kTokenBytes / 16;
  const uint32_t sb = sa + 4 * T::kAtoms;
#pragma unroll
  for (int atom = 0; atom < STEPS / per; ++atom) {
    copy_scales<1>(sa + 4 * atom, sc + atom * (kAtomBytes / 16));
    copy_scales<1>(sb + 4 * atom, sc + ((T::kScales - 1) * T::kScaleBytes + atom * kAtomBytes) / 16);
  }
#pragma unroll
  for (int j = 0; j < STEPS; ++j) {
    const int atom = j / per;
    mma<GROUP, 1>(acc, src + 2 * j, tokens + 2 * j, instruction<GROUP>(128, BN, GROUP == 32 ? 2 * (j % 2) : 0), sa + 4 * atom,
                  sb + 4 * atom, j > 0 || !fresh);
  }
}

// A gated tile's scales: of every line of 16 bytes (4 words, 32 rows apart) the gate's two words of this half of 128 features
// and then the up projection's two, in the gate's place.
template <int BYTES>
__device__ __forceinline__ void mix_scales(uint32_t gate, uint32_t up, bool upper, int lane) {
#pragma unroll
  for (int i = 0; i < BYTES; i += 512) {
    const uint32_t half = uint32_t(i + lane * 16) + (upper ? 8u : 0u);
    uint32_t g0, g1, u0, u1;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(g0), "=r"(g1) : "r"(gate + half) : "memory");
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(u0), "=r"(u1) : "r"(up + half) : "memory");
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(gate + uint32_t(i + lane * 16)), "r"(g0), "r"(g1), "r"(u0), "r"(u1)
                 : "memory");
  }
}

template <int GROUP, int BN, int MODE>
__global__ void __launch_bounds__(kStreamThreads, 2)
mx_stream_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_u,
                 const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_sw,
                 const __grid_constant__ CUtensorMap map_su, const __grid_constant__ CUtensorMap map_sx, const Args p,
                 const int parts) {
  constexpr bool GATED = MODE != kLinear;
  using T = Stream<GROUP, BN, GATED>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t base = (raw_addr + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (base - raw_addr);
  const uint32_t bar_base = base + T::kRingBytes;
  auto full = [&](int s) { return bar_base + 8u * s; };
  auto empty = [&](int s) { return bar_base + 8u * (T::kStages + s); };
  auto mixed = [&](int s) { return bar_base + 8u * (2 * T::kStages + s); };      // gated tiles' scales
  const uint32_t done = bar_base + 8u * (T::kBarriers - 1);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + T::kRingBytes + 8 * T::kBarriers);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = warp_number(), lane = threadIdx.x & 31;
  const int part = int(blockIdx.x) % parts;                 // rank in the cluster
  const int tile = int(blockIdx.x) / parts;
  const int m0 = int(blockIdx.y) * BN, n0 = tile * T::kTileRows;
  const int k0 = int(int64_t(p.kblocks) * part / parts), k1 = int(int64_t(p.kblocks) * (part + 1) / parts);
  if (parts > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");     // this CTA runs: its memory may be written
  const int slots = (BN + parts - 1) / parts;               // tokens that a CTA finishes, at the most
  const uint32_t sums_at = parts > 1 ? base + uint32_t(T::kRingBytes + T::kHeadBytes) : base;
  auto set_up = [] { asm volatile("bar.sync 1, %0;" ::"n"(kStreamThreads) : "memory"); };
  // Warp 0 sets up the barriers and has loads on their way before the others have their tensor memory.
  if (warp == 0) {
    const bool one = elected();
    if (one) {
      for (int s = 0; s < T::kStages; ++s) {
        bar_init(full(s), 1);
        bar_init(empty(s), 1);
        if (GATED) bar_init(mixed(s), 1);
      }
      bar_init(done, 1);
      *abort_flag = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      fence_async();
    }
    __syncwarp();
    after_the_call_before();
    Ring<T::kStages> r;
    for (int kb = k0; kb < k1; ++kb, r.next()) {
      if (kb == k0 + T::kStages) set_up();       // the others may go on: the ring's first round is under way
      if (!bar_wait_warp(empty(r.s), r.phase ^ 1u, abort_flag, kStreamLoad)) break;
      if (one) {
        const uint32_t bar = full(r.s);
        bar_expect(bar, uint32_t(T::kStageBytes));
        const uint32_t dst = base + r.s * T::kStageBytes, sc = dst + kTileBytes + T::kTokenBytes;
        const int x = kb * (T::kScaleBytes / 8);
        tma_load(dst, &map_w, bar, kb * kRowBytes, n0);
        if (GATED) tma_load(dst + kTileBytes / 2, &map_u, bar, kb * kRowBytes, n0);
        tma_load(dst + kTileBytes, &map_x, bar, kb * kRowBytes, m0);
        tma_load(sc, &map_sw, bar, x, n0 / kTile);
        if (GATED) tma_load(sc + T::kScaleBytes, &map_su, bar, x, n0 / kTile);
        tma_load(sc + (T::kScales - 1) * T::kScaleBytes, &map_sx, bar, x, m0 / kTile);
      }
      __syncwarp();
    }
    if (k1 - k0 <= T::kStages) set_up();
  } else {
    if (warp == 1) tmem_alloc<1>(smem_u32(tmem_slot), T::kTmemCols);
    if (warp == 3 && blockIdx.y == 0 && elected()) {
      // While the call before finishes, the first weights are asked into L2 (no further: that one may be asking for its own; two
      // k-blocks were 3 % faster than none over 40 calls with weights from memory, four 2.6 %).
      for (int kb = k0; kb < min(k1, k0 + 2); ++kb) {
        const int x = kb * (T::kScaleBytes / 8);
        tma_prefetch(&map_w, kb * kRowBytes, n0);
        tma_prefetch(&map_sw, x, n0 / kTile);
        if (GATED) tma_prefetch(&map_u, kb * kRowBytes, n0);
        if (GATED) tma_prefetch(&map_su, x, n0 / kTile);
      }
    }
    __syncwarp();
    after_the_call_before();
    fence_before();
    set_up();
    fence_after();
  }
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);       // in warp 0, which has no use for it, anything

  if (warp == 1) {
    const bool one = elected();
    const uint32_t sa = tmem + T::kScaleCol;
    Ring<T::kStages> r;
    bool ok = true;
    for (int kb = k0; kb < k1; ++kb, r.next()) {
      ok = bar_wait_warp(full(r.s), r.phase, abort_flag, kStreamFull);
      if (GATED) ok = ok && bar_wait_warp(mixed(r.s), r.phase, abort_flag, kStreamMixed);
      if (!ok) break;
      fence_after();
      if (one) {
        const uint32_t src = desc_low(base + r.s * T::kStageBytes);
        if (kb + 1 < p.kblocks || p.last_steps == kStepsPerBlock)
          stream_block<GROUP, BN, GATED, kStepsPerBlock>(tmem, src, sa, kb == k0);
        else
          stream_block<GROUP, BN, GATED, kStepsPerBlock / 2>(tmem, src, sa, kb == k0);
        commit(empty(r.s));
      }
      __syncwarp();
    }
    if (ok && one) commit(done);
    __syncwarp();
  } else if (GATED && warp == 2) {
    Ring<T::kStages> r;
    for (int kb = k0; kb < k1; ++kb, r.next()) {
      if (!bar_wait_warp(full(r.s), r.phase, abort_flag, kStreamMixed)) break;
      const uint32_t sc = base + r.s * T::kStageBytes + kTileBytes + T::kTokenBytes;
      mix_scales<T::kScaleBytes>(sc, sc + T::kScaleBytes, (tile & 1) != 0, lane);
      fence_async();
      __syncwarp();
      if (lane == 0) bar_arrive_cluster(mixed(r.s));
    }
  }
  __syncwarp();
  // What the end needs of the steps is asked for meanwhile: a thread finishes 8 neighbouring channels of tokens, so that 4 lanes hold a
  // group or rotation block of 32.  The tokens' steps as far as the SM's cache.
  constexpr int kChunks = T::kTileRows / 8;
  const int f = int(threadIdx.x) - 64, chunk = f % kChunks, n = n0 + chunk * 8;
  const bool on = n < p.N;
  float ws[8], us[8];
  if (warp >= 2) {
    eight_steps(on ? p.w_step : nullptr, n, ws);
    if (GATED) eight_steps(on ? p.up_step : nullptr, n, us);
    if (f < BN && m0 + f < p.M) {
      if (p.x_step != nullptr) (void)load(p.x_step + m0 + f);
      if (MODE == kGatedCodes && GROUP == 16) (void)load(p.h_step + m0 + f);
    }
  }
  if (parts > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (warp >= 2 && bar_wait_warp(done, 0, abort_flag, kStreamEpilogue)) {
    // [part][token][row of the tile] of the tokens that a CTA finishes: token c is the c / parts th of CTA c % parts
    fence_after();
    const int q = warp & 3, half = (warp - 2) >> 2;
    const uint32_t acc = tmem + (uint32_t(q * 32) << 16);
    const uint32_t to = sums_at + uint32_t((part * slots * kTile + q * 32 + lane) * 4);
    const int cols = min(BN, p.M - m0), shift = 31 - __clz(parts);
    constexpr int kRead = BN >= 32 ? 16 : 8;       // tokens at a time
#pragma unroll 1
    for (int c = half * kRead; c < cols; c += 2 * kRead) {
      float v[kRead];
      tmem_load(acc + c, v);
      tmem_wait_ld();
      auto send = [&](auto quotient_of, auto rest_of) {
#pragma unroll
        for (int i = 0; i < kRead; ++i)
          asm volatile("st.shared::cluster.f32 [%0], %1;"
                       ::"r"(map_to_cta(to + uint32_t(quotient_of(c + i) * kTile * 4), uint32_t(rest_of(c + i)))), "f"(v[i]) : "memory");
      };
      if (parts == 1) {
#pragma unroll
        for (int i = 0; i < kRead; ++i) asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + uint32_t((c + i) * kTile * 4)), "f"(v[i]) : "memory");
      } else if (parts == 3) {
        send([](int t) { return (t * 342) >> 10; }, [](int t) { return t - ((t * 342) >> 10) * 3; });      // t / 3, t % 3 for t < 512
      } else {
        send([&](int t) { return t >> shift; }, [&](int t) { return t & (parts - 1); });
      }
    }
  }
  drain_after_abort(abort_flag);
  fence_before();
  __syncwarp();
  if (parts > 1) cluster_sync();
  else __syncthreads();
  if (*abort_flag == 0 && warp >= 2) {
    // This CTA's tokens are m0 + part, m0 + part + parts, ..  All lanes of a warp take part; those past the last token repeat it and
    // write nothing.
    const int cols = min(BN, p.M - m0), mine = (cols - part + parts - 1) / parts;
    for (int i0 = warp_number() * 32 - 64; i0 / kChunks < mine; i0 += 256) {
      const int i = (i0 + lane) / kChunks;
      const bool there = i < mine && on;
      const int c = min(i, mine - 1) * parts + part, m = m0 + c;
      float a[8], b[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) a[j] = b[j] = 0.0f;
      uint32_t at = sums_at + uint32_t((min(i, mine - 1) * kTile + chunk * 8) * 4);
      for (int r = 0; r < parts; ++r, at += uint32_t(slots * kTile * 4)) {
        add_shared(a, at);
        if (GATED) add_shared(b, at + uint32_t(kTile / 2 * 4));
      }
      const float xs = p.x_step != nullptr ? load(p.x_step + m) : 1.0f;
      const f32x2 xs2 = pack2(xs, xs);
      f32x2 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = mul2(pack2(a[2 * j], a[2 * j + 1]), mul2(xs2, pack2(ws[2 * j], ws[2 * j + 1])));
        if constexpr (GATED) {
          const f32x2 up = mul2(pack2(b[2 * j], b[2 * j + 1]), mul2(xs2, pack2(us[2 * j], us[2 * j + 1])));
          v[j] = MODE == kGatedCodes ? silu_exact(v[j], up) : silu_times(v[j], up);
        }
      }
      if (GATED && p.walsh) walsh_rows<32>(v, p.norm, lane);
      if constexpr (MODE == kGatedCodes) {
        uint32_t byte;
        const RowStep row = GROUP == 16 ? row_step(load(p.h_step + m)) : RowStep{};
        const Part<1> codes = encode<GROUP, true>(v, top_of(v), row, &byte);
        if (there) {
          *reinterpret_cast<uint32_t*>(p.q_out + int64_t(m) * (p.N / 2) + n / 2) = codes.w[0];
          if (writes_scale<GROUP, 4>(chunk))
            p.scale_out[scale_word(m, 0, p.N / (4 * GROUP)) + scale_offset<GROUP, 4>(n / 8)] = uint8_t(byte);
        }
      } else {
        const Part<4> h = narrow(v);
        if (there) *reinterpret_cast<uint4*>(p.y + int64_t(m) * p.ldy + n) = make_uint4(h.w[0], h.w[1], h.w[2], h.w[3]);
      }
    }
  }
  if (warp == 1) {
    __syncwarp();
    fence_after();
    tmem_free<1>(tmem, T::kTmemCols);
  }
}

// Test probe: one warp waits, through the kernels' bounded wait, on a barrier that nobody arrives on.
__global__ void mx_wait_probe_kernel() {
  __shared__ __align__(8) unsigned long long storage;
  __shared__ int abort_word;
  const uint32_t bar = smem_u32(&storage);
  if (threadIdx.x == 0) {
    abort_word = 0;
    bar_init(bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  (void)bar_wait(bar, 0u, &abort_word, kProbe);
  drain_after_abort(&abort_word);
}

// ---- host ----

// Packed codes [rows x K/2] bytes, `box` rows of 128 bytes at a time, 128-byte swizzle.  Past the edges: zeros.
bool map_codes(CUtensorMap* map, const uint8_t* p, int64_t rows, int64_t K, int box) {
  const cuuint64_t dims[2] = {cuuint64_t(K / 2), cuuint64_t(rows)};
  const cuuint64_t strides[1] = {cuuint64_t(K / 2)};
  const cuuint32_t boxes[2] = {kRowBytes, cuuint32_t(box)}, ones[2] = {1, 1};
  return tensor_map_encoder()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(p), dims, strides, boxes, ones,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Blocks of scales, 8 bytes an element: those of 128 rows in a line, a k-block's at a time.
bool map_scales(CUtensorMap* map, const uint8_t* p, int64_t rows, int64_t K, int group) {
  const int64_t quads = K / group / kAtomGroups;
  const cuuint64_t dims[2] = {cuuint64_t(quads * (kAtomBytes / 8)), cuuint64_t((rows + kAtomRows - 1) / kAtomRows)};
  const cuuint64_t strides[1] = {cuuint64_t(quads * kAtomBytes)};
  const cuuint32_t boxes[2] = {cuuint32_t(kBlockK / group / kAtomGroups * (kAtomBytes / 8)), 1}, ones[2] = {1, 1};
  return tensor_map_encoder()(map, CU_TENSOR_MAP_DATA_TYPE_INT64, 2, const_cast<uint8_t*>(p), dims, strides, boxes, ones,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// fp16 output [M x N], boxes of 32 rows and 32 columns for stores.
bool map_half(CUtensorMap* map, __half* y, int64_t M, int64_t N, int64_t ldy) {
  const cuuint64_t dims[2] = {cuuint64_t(N), cuuint64_t(M)};
  const cuuint64_t strides[1] = {cuuint64_t(ldy) * sizeof(__half)};
  const cuuint32_t boxes[2] = {32, 32}, ones[2] = {1, 1};
  return tensor_map_encoder()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, y, dims, strides, boxes, ones,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
                              CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Call {
  const uint8_t *x, *sx, *w, *sw, *u, *su;
  int64_t M, N, K;
  Args args;
  cudaStream_t stream;
};

template <int GROUP, int MODE>
int launch_pair(const Call& c) {
  using T = Pair<GROUP>;
  constexpr bool gated = MODE != kLinear;
  CUtensorMap a, b, u, sa, sb, su, y;
  if (!map_codes(&a, c.x, c.M, c.K, kTile) || !map_codes(&b, c.w, c.N, c.K, kTile) ||
      !map_scales(&sa, c.sx, c.M, c.K, GROUP) || !map_scales(&sb, c.sw, c.N, c.K, GROUP))
    return SMOOTHROT_CUDA_ERROR;
  u = b;
  su = sb;
  if (gated && (!map_codes(&u, c.u, c.N, c.K, kTile) || !map_scales(&su, c.su, c.N, c.K, GROUP))) return SMOOTHROT_CUDA_ERROR;
  y = a;
  if (MODE != kGatedCodes && !map_half(&y, c.args.y, c.M, c.N, c.args.ldy)) return SMOOTHROT_CUDA_ERROR;
  Args p = c.args;
  const int width = gated ? kTile : 256;
  p.tiles_a = int((c.M + 255) / 256);
  p.tiles_b = int((c.N + width - 1) / width);
  auto kern = mx_pair_kernel<GROUP, MODE>;
  if (!allow_dynamic_smem(reinterpret_cast<const void*>(kern), T::kSmemBytes)) return SMOOTHROT_CUDA_ERROR;
  const int64_t tiles = int64_t(p.tiles_a) * p.tiles_b, pairs = device_sm_count() / 2;
  return launch(kern, dim3(unsigned(2 * (tiles < pairs ? tiles : pairs))), T::kThreads, T::kSmemBytes, 0, c.stream, a, b, u, sa, sb, su,
                y, p);
}

template <int GROUP, int BN, int MODE>
int launch_stream(const Call& c, int parts) {
  using T = Stream<GROUP, BN, MODE != kLinear>;
  CUtensorMap w, u, x, sw, su, sx;
  if (!map_codes(&w, c.w, c.N, c.K, T::kTileRows) || !map_codes(&x, c.x, c.M, c.K, BN) ||
      !map_scales(&sw, c.sw, c.N, c.K, GROUP) || !map_scales(&sx, c.sx, c.M, c.K, GROUP))
    return SMOOTHROT_CUDA_ERROR;
  u = w;
  su = sw;
  if (MODE != kLinear && (!map_codes(&u, c.u, c.N, c.K, T::kTileRows) || !map_scales(&su, c.su, c.N, c.K, GROUP)))
    return SMOOTHROT_CUDA_ERROR;
  auto kern = mx_stream_kernel<GROUP, BN, MODE>;
  if (!allow_dynamic_smem(reinterpret_cast<const void*>(kern), T::kSmemBytes + T::kSumBytes)) return SMOOTHROT_CUDA_ERROR;
  const dim3 grid(unsigned((c.N + T::kTileRows - 1) / T::kTileRows * parts), unsigned((c.M + BN - 1) / BN));
  return launch(kern, grid, kStreamThreads, T::kSmemBytes + (parts > 1 ? T::kSumBytes : 0), parts, c.stream, w, u, x, sw, su, sx, c.args, parts);
}

// Clusters of `size` CTAs, one to an SM, that the device runs at once: a cluster stays inside a part of the chip, so large ones
// leave SMs over (148, 74, 33, 15 of 1, 2, 4, 8 on B200).  Asked of the runtime once per device, for the form with the most tokens, of which
// one CTA fits an SM as of nearly all that are split.
int clusters_at_once(int size) {
  constexpr int kDevices = 64, kMostParts = 8;
  static std::atomic<int> known[kDevices][kMostParts + 1];
  int dev = 0;
  if (size > kMostParts || cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return device_sm_count() / (size * 2);
  int n = known[dev][size].load(std::memory_order_relaxed);
  if (n > 0) return n;
  typedef Stream<32, 128, false> T;
  auto kern = mx_stream_kernel<32, 128, kLinear>;
  const int bytes = T::kSmemBytes + T::kSumBytes;
  if (allow_dynamic_smem(reinterpret_cast<const void*>(kern), bytes)) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(size * 32), 1, 1);
    cfg.blockDim = dim3(kStreamThreads, 1, 1);
    cfg.dynamicSmemBytes = size_t(bytes);
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = unsigned(size);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) n = 0;
  }
  if (n <= 0) {
    (void)cudaGetLastError();
    return device_sm_count() / (size * 2);
  }
  known[dev][size].store(n, std::memory_order_relaxed);
  return n;
}

// Which kernel.  Up to 128 tokens the few-token one was the faster at every size tried (1 x 4096 x 4096: 4.1 us against 8.5; 128 x
// 6144 x 4096: 8.3 against 9.9; gated 14336 x 4096: 13.2 against 22.6 with one token, 16.6 against 18.4 with 128).  K is split over
// as many CTAs as leave every tile's cluster a place at once (61 x 5120 x 4096 in 3 parts 6.2 us, in 2 6.5; 4096 x 14336 in 4
// 9.3, in 2 12.5, in 8, not all at once, 18.7).
// Beyond 128 tokens an estimate decides, in us: a fixed part, then a time per k-block and wave of tiles; scales of groups of 16, twice as
// many, weigh on the few-token kernel.  Measured, few-token | pair: 256 x 4096 x 14336 15.9 | 21.5, 200 x 2048 x 5632 7.0 | 11.1, 512 x
// 4096 x 4096 10.3 | 9.9.  Gated into codes: 200 x 1408 x 2048 6.3 | 7.1, 300 x 5632 x 2048 10.6 | 10.7, in groups of 16 13.1 | 12.5,
// 200 x 5632 x 2048 10.2 | 8.1.
template <int GROUP, int MODE>
int run(const Call& c) {
  constexpr bool gated = MODE != kLinear;
  const int64_t rows = gated ? kTile / 2 : kTile, tiles = (c.N + rows - 1) / rows * ((c.M + 127) / 128);
  int parts = 1;
  for (int more : {2, 3, 4, 8}) {
    if (c.args.kblocks < more || tiles > clusters_at_once(more)) break;
    parts = more;
  }
  if (c.M > 128) {
    const int width = gated ? kTile : 256;
    const int64_t sms = device_sm_count(), pairs = sms / 2, ctas = tiles * parts;
    const double waves = double(((c.M + 255) / 256 * ((c.N + width - 1) / width) + pairs - 1) / pairs);
    const double blocks = double((c.args.kblocks + parts - 1) / parts);
    double pair_us, stream_us;
    if (gated) {
      const double each = (ctas <= sms ? 0.5 : 0.67 * double((ctas + 2 * sms - 1) / (2 * sms))) * (GROUP == 16 ? 1.45 : 1.0);
      pair_us = 5.4 + 0.33 * double(c.args.kblocks) * waves;
      stream_us = 5.0 + blocks * each;
    } else {
      pair_us = 4.6 + 0.30 * double(c.args.kblocks) * waves;
      stream_us = 4.6 + blocks * 0.38 * (ctas > sms ? double(ctas) / double(sms) : 1.0);
    }
    return stream_us < pair_us ? launch_stream<GROUP, 128, MODE>(c, parts) : launch_pair<GROUP, MODE>(c);
  }
  if (c.M <= 16) return launch_stream<GROUP, 16, MODE>(c, parts);
  if (c.M <= 32) return launch_stream<GROUP, 32, MODE>(c, parts);
  if (c.M <= 64) return launch_stream<GROUP, 64, MODE>(c, parts);
  return launch_stream<GROUP, 128, MODE>(c, parts);
}

int check_operand(const uint8_t* q, const uint8_t* s) {
  if (q == nullptr || s == nullptr) return SMOOTHROT_INVALID_ARG;
  return aligned16(q) && aligned16(s) ? SMOOTHROT_OK : SMOOTHROT_BAD_ALIGNMENT;
}

// a step per row, read four at a time where it is the weights'
bool bad_steps(std::initializer_list<const float*> steps) {
  for (const float* p : steps)
    if (p != nullptr && !aligned16(p)) return true;
  return false;
}

int check_sizes(int64_t M, int64_t N, int64_t K, int64_t group) {
  if (M < 0 || N < 0 || K <= 0 || !group_ok(group)) return SMOOTHROT_INVALID_ARG;
  if (K % 128 != 0 || K > (int64_t(1) << 20)) return SMOOTHROT_UNSUPPORTED_K;
  if (N % 8 != 0 || M > 0x7fffffffLL / 2 || N > 0x7fffffffLL / 2) return SMOOTHROT_INVALID_ARG;
  return SMOOTHROT_OK;
}

}  // namespace
}  // namespace mx
}  // namespace smoothrot

extern "C" {

int smoothrot_mx_status_word(int* out, int clear) {
  int rc = smoothrot::mx::read_status_word(smoothrot::mx::g_mx_status, out, clear), norm = 0;
  if (rc == SMOOTHROT_OK) rc = smoothrot_norm_status_word(&norm, clear);
  if (*out == 0) *out = norm;
  return rc;
}

int smoothrot_mx_set_wait_limit_ns(uint64_t ns) {
  const unsigned long long v = ns == 0 ? smoothrot::mx::kWaitLimitNs : static_cast<unsigned long long>(ns);
  if (cudaMemcpyToSymbol(smoothrot::mx::g_mx_wait_limit_ns, &v, sizeof(v)) != cudaSuccess) return SMOOTHROT_CUDA_ERROR;
  return smoothrot_norm_set_wait_limit_ns(ns);
}

int smoothrot_debug_mx_wait_expiry(void* stream) {
  smoothrot::mx::mx_wait_probe_kernel<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>();
  smoothrot::count_launch();
  return smoothrot::launch_status();
}

int smoothrot_mx_linear(const uint8_t* Xq, const uint8_t* x_scale, const float* x_step, int64_t M, const uint8_t* Wq,
                        const uint8_t* w_scale, const float* w_step, int64_t N, int64_t K, int64_t group, void* Y_f16,
                        int64_t ldy, void* stream) {
  using namespace smoothrot;
  using namespace smoothrot::mx;
  int rc = check_sizes(M, N, K, group);
  if (rc != SMOOTHROT_OK || M == 0 || N == 0) return rc;
  if (Y_f16 == nullptr || ldy < N) return SMOOTHROT_INVALID_ARG;
  if ((rc = check_operand(Xq, x_scale)) != SMOOTHROT_OK || (rc = check_operand(Wq, w_scale)) != SMOOTHROT_OK) return rc;
  if (!aligned16(Y_f16) || ldy % 8 != 0 || bad_steps({w_step})) return SMOOTHROT_BAD_ALIGNMENT;
  if (tensor_map_encoder() == nullptr) return SMOOTHROT_CUDA_ERROR;
  Call c{Xq, x_scale, Wq, w_scale, nullptr, nullptr, M, N, K, Args{}, static_cast<cudaStream_t>(stream)};
  c.args.M = int(M);
  c.args.N = int(N);
  c.args.kblocks = int((K + kBlockK - 1) / kBlockK);
  c.args.last_steps = K % kBlockK == 0 ? kStepsPerBlock : kStepsPerBlock / 2;
  c.args.x_step = x_step;
  c.args.w_step = w_step;
  c.args.y = static_cast<__half*>(Y_f16);
  c.args.ldy = ldy;
  return group == 32 ? run<32, kLinear>(c) : run<16, kLinear>(c);
}

int smoothrot_mx_glu(const uint8_t* Xq, const uint8_t* x_scale, const float* x_step, int64_t M, const uint8_t* gate_q,
                     const uint8_t* gate_scale, const float* gate_step, const uint8_t* up_q, const uint8_t* up_scale,
                     const float* up_step, int64_t F, int64_t K, int64_t group, int walsh, void* H_f16, int64_t ldh,
                     uint8_t* q_out, uint8_t* scale_out, const float* h_step, void* stream) {
  using namespace smoothrot;
  using namespace smoothrot::mx;
  int rc = check_sizes(M, F, K, group);
  if (rc != SMOOTHROT_OK) return rc;
  if (walsh != 0 && walsh != 32) return SMOOTHROT_INVALID_ARG;
  const bool codes = q_out != nullptr;
  if ((codes && F % 128 != 0) || (walsh != 0 && F % 32 != 0)) return SMOOTHROT_UNSUPPORTED_K;
  if (M == 0 || F == 0) return SMOOTHROT_OK;
  if (codes == (H_f16 != nullptr)) return SMOOTHROT_INVALID_ARG;      // one of the two forms
  if (codes && (scale_out == nullptr || (group == 16) != (h_step != nullptr))) return SMOOTHROT_INVALID_ARG;
  if (!codes && (ldh < F || scale_out != nullptr || h_step != nullptr)) return SMOOTHROT_INVALID_ARG;
  if ((rc = check_operand(Xq, x_scale)) != SMOOTHROT_OK || (rc = check_operand(gate_q, gate_scale)) != SMOOTHROT_OK ||
      (rc = check_operand(up_q, up_scale)) != SMOOTHROT_OK)
    return rc;
  if (codes ? !aligned16(q_out) || !aligned16(scale_out) : !aligned16(H_f16) || ldh % 8 != 0) return SMOOTHROT_BAD_ALIGNMENT;
  if (bad_steps({gate_step, up_step})) return SMOOTHROT_BAD_ALIGNMENT;
  if (tensor_map_encoder() == nullptr) return SMOOTHROT_CUDA_ERROR;
  Call c{Xq, x_scale, gate_q, gate_scale, up_q, up_scale, M, F, K, Args{}, static_cast<cudaStream_t>(stream)};
  c.args.M = int(M);
  c.args.N = int(F);
  c.args.kblocks = int((K + kBlockK - 1) / kBlockK);
  c.args.last_steps = K % kBlockK == 0 ? kStepsPerBlock : kStepsPerBlock / 2;
  c.args.x_step = x_step;
  c.args.w_step = gate_step;
  c.args.up_step = up_step;
  c.args.y = static_cast<__half*>(H_f16);
  c.args.ldy = ldh;
  c.args.q_out = q_out;
  c.args.scale_out = scale_out;
  c.args.h_step = h_step;
  c.args.walsh = walsh;
  c.args.norm = walsh != 0 ? float(1.0 / sqrt(double(walsh))) : 1.0f;
  if (codes) return group == 32 ? run<32, kGatedCodes>(c) : run<16, kGatedCodes>(c);
  return group == 32 ? run<32, kGatedHalf>(c) : run<16, kGatedHalf>(c);
}

}  // extern "C"
