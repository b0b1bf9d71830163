// Attention of one new token per sequence over the paged key-value cache (layout: paged.cuh).
//
//   y = sum_j p_j v_j / sum_j p_j,   p_j = 2^(x_j - m),   x_j = scale log2(e) q.k_j
//
// The cache is read once, and that bounds the kernel: 4-bit keys and values of a head of 128 are 144
// bytes a token, for 4 D flops per query head.
//
// Work: a segment is one sequence and one key head with up to 8 (or 16) of its query heads.  All
// segments' tiles of keys stand in one line, and every warp takes an equal stretch of it, whatever the lengths.  A
// segment that lies within a stretch is finished by its warp; pieces of one meet in shared memory, and
// where a segment reaches over several CTAs, in the workspace: the last CTA to arrive adds the
// pieces up, in the order of the tiles, so the result does not depend on who came last.
//
// A warp streams its tiles through a ring of its own (bulk copies, a lane for each run of rows in one page; no barrier
// with other warps) and computes with the
// warp-level matrix instruction (m16n8k16): the keys of a tile are the 16 rows, the query heads the 8 columns, so a group of
// 4 or 8 heads wastes little, where the tensor-memory instructions would want 128 rows:
//     S^T [keys x heads] = K Q^T,   O^T [values x heads] += V^T P^T
// P leaves S's registers for the second product through movmatrix.  4-bit codes become fp16 whole numbers (exact) in
// registers; step and zero point are applied to the small side:
//     x = (q.c - z sum(q)) s_k,   O = sum w c - sum w z,   w = p s_v
// The weight w is rounded once to fp16, and both sums take the rounded one (the denominator sums p before it is rounded).  So that w fits fp16 whatever the
// step, the reference m runs over x + log2(s_v); p itself, summed in fp32 for the denominator, may then exceed 1.
// m is set so that the largest w is 2^7 and raised only where one exceeds 2^15, half of what fp16 holds: most tiles need no
// exchange between lanes, and a weight keeps its 11 bits down to 2^-21 of the largest and counts down to 2^-31 (small weights
// of many keys add up).  Steps of one sequence that differ by more than 2^21 cost the smaller ones bits.  A group of equal
// values has the step 1, so a row of zeros would set the reference for values of any size: where one asks for a higher
// reference its step is taken as 2^-60, which leaves its value what it is.
//
// Measured (device time; floor at 6552 GB/s in brackets): 32 query and 8 key heads of 128, 4 bits: one sequence of 131072
// tokens 47.9 us (23.0), 64 of up to 4001 55.3 us (23.5), one of 301 9.6 us; 16 of up to 2048 with 32 fp16 heads 61 us
// (43).  Pages are of 16 tokens in all but the first (64); the 64 sequences take 157 us with pages of 1, 108 with 2, 69 with 4,
// 60 with 8, 54 with 256 and more: a tile is then several copies, and with fewer than 4 tokens a page more than one a lane.
// The copies alone, without any arithmetic, take 39 us of the 48: about 4.5 us until the first tile is asked for, 26
// of streaming, 7 to join the pieces (each step of which waits for memory: flags 2, their pieces 3).  The arithmetic
// adds 9: a tile of 32 keys is 600 instructions, 290 of them on the ALU at half rate, for 790 cycles of a scheduler at
// the memory's pace, and four warps a scheduler reach half of its slots.  With fp16 values the loop runs at the memory's
// rate.  Few registers and many warps matter more than anything else here: 128 registers and 16 warps beat 168 and
// 12 (59), 96 and 20 (62), and scores of one tile beside values of the last (61).
#include "paged.cuh"
#include "rowquant.cuh"

// defined with the attention over prompts: a probe of its waits
extern "C" int smoothrot_prefill_wait_expiry(int site, void* stream);

namespace smoothrot {
namespace paged {

__device__ int g_decode_status = 0;
constexpr unsigned long long kDecodeWaitLimitNs = 2000000000ull;
__device__ unsigned long long g_decode_wait_limit_ns = kDecodeWaitLimitNs;
constexpr unsigned long long kAtOnceNs = 1000;   // a limit below this is taken as run out before the first copy (for tests: no copy is
                                                 // late by itself, and a single try waits longer)
constexpr unsigned long long kDecodeDrainNs = 1000000ull;
constexpr int kDecodeWait = 41;
constexpr uint32_t kGaveUp = 1u << 31;           // in a warp's phases: a wait ran out, nothing more is loaded
constexpr uint32_t kNoKey = 1u << 30;            // every token of this piece so far was left out

constexpr int kWarps = 8;
constexpr int kDecodeThreads = 32 * kWarps;
static_assert(2 * kWarps <= 16, "two records a warp, found by half a warp");

struct DecodeArgs {
  const __half* q;
  int64_t ldq;
  const int32_t* table;     // [batch][max_pages]
  int64_t max_pages;
  const int32_t* lengths;
  __half* y;
  int64_t ldy;
  int batch;
  int group;                // query heads per key head
  int rows;                 // of them in a segment
  int chunks;               // segments per key head
  int units;                // segments per sequence
  float c;                  // scale log2(e)
  unsigned long long* arrived;   // [grid][2]
  float* records;           // [grid][2][rows * D + 2 * rows]
  unsigned long long tag;   // of this call, even and not 0
};

template <int D, int kBits, int NT>
struct Shape {
  static constexpr int kKeys = kBits == 4 ? 32 : 16;                 // of a tile
  static constexpr int kRowBytes = kBits == 4 ? D / 2 : 2 * D;
  static constexpr int kStageBytes = 2 * kKeys * kRowBytes + (kBits == 4 ? 2 * kKeys * 8 : 0);
  static constexpr int kStages = kBits == 4 ? 2 : (D == 64 ? 4 : (NT == 1 ? 3 : 2));
  static constexpr int kRingBytes = kStages * kStageBytes;           // of a warp
  static constexpr int kCtas = kBits == 4 && NT == 1 ? 2 : 1;        // resident per SM
  static constexpr int kRecord = 8 * NT * (D + 2);                   // floats, at most
  // a warp's second record goes over its ring, when that is done with
  // (the weights of the pieces of a segment, 16 floats for each of 2 x 160 CTAs at most, fit over all of them)
  static constexpr int kWarpBytes = kRingBytes > kRecord * 4 ? kRingBytes : kRecord * 4;
};

struct Segment {
  int b, unit, tile, tiles, length;
};

__device__ __forceinline__ int clamped_length(const DecodeArgs& a, const Cache& c, int b) {
  const int n = a.lengths[b];
  const int64_t most = a.max_pages << c.page_shift;
  return n < 0 ? 0 : (n > most ? int(most) : n);
}

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_rows(uint32_t dst, const void* src, uint32_t size, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(size), "r"(bar)
               : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
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
// Wait of a whole warp for a stage's copies, bounded; false (in every lane) if it ran out.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  bool ok = bar_try(bar, parity);
  if (!__all_sync(0xffffffffu, ok)) {
    const unsigned long long t0 = now_ns();
    while (!ok && now_ns() - t0 <= g_decode_wait_limit_ns) ok = bar_try(bar, parity);
    return __all_sync(0xffffffffu, ok);
  }
  return true;
}

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float log2_fast(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }

// Codes k and k + 4 of a word (k = 0 .. 3), less 8, as two fp16 whole numbers.  0x6400 is 1024 in fp16 with a last place
// of 1, so a code or-ed into it is 1024 + code; four places higher it counts 16 times.  The 8 comes off the zero point
// too: sums of codes around zero are small, and what the tensor core cuts off their last places with them.
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t (&h)[4]) {
  const uint32_t up = w >> 8;
  uint32_t x[4];
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(x[0]) : "r"(w));
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x64006400, 0xEA;" : "=r"(x[1]) : "r"(w));
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(x[2]) : "r"(up));
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x64006400, 0xEA;" : "=r"(x[3]) : "r"(up));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(h[0]) : "r"(x[0]), "r"(0x64086408u));
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(h[1]) : "r"(x[1]), "r"(0x2C002C00u), "r"(0xD480D480u));   // x / 16 - 72
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(h[2]) : "r"(x[2]), "r"(0x64086408u));
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(h[3]) : "r"(x[3]), "r"(0x2C002C00u), "r"(0xD480D480u));
}

// The same for keys: a code in bits 4..7 over 0x5400 is 64 + code (last place 1/16), which saves the second
// operation; the 72 = 64 + 8 too many of the odd codes are taken off the score before its sum starts.
__device__ __forceinline__ void key_codes_to_half(uint32_t w, uint32_t (&h)[4]) {
  const uint32_t up = w >> 8;
  uint32_t x[2];
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(x[0]) : "r"(w));
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x54005400, 0xEA;" : "=r"(h[1]) : "r"(w));
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(x[1]) : "r"(up));
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x54005400, 0xEA;" : "=r"(h[3]) : "r"(up));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(h[0]) : "r"(x[0]), "r"(0x64086408u));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(h[2]) : "r"(x[1]), "r"(0x64086408u));
}

// Key of a tile's 16 that stands in row r of the first product, and so in place r of the second's sum.  A lane's
// four places 2t, 2t+1, 2t+8, 2t+9 of the sum are then rows t, 4 + (t^1), 8 + t, 12 + (t^1): the four lanes of one read
// cover whole rows of values, and two neighbouring rows of keys start in different halves of a 128-byte line.
__device__ __forceinline__ int key_of_row(int r) {
  const int t = (r & 7) >> 1;
  return (r & 8) + ((r & 1) ? 4 + (t ^ 1) : t);
}

constexpr float kNoMaximum = 3e38f;              // -m before the first key: exceeded by any finite score
constexpr float kStepOfZeros = 8.673617379884035e-19f;     // 2^-60: neither its weight nor the sum of the p overflows

template <int D, int kBits, int NT>
struct Piece {                                   // what a warp has of a segment
  float o[D / 16][NT][4];                        // [pairs of values][8 heads][(value 2i, head 2t), (2i, 2t+1), (2i+1, 2t), (2i+1, 2t+1)]
  f32x2 neg_m[NT], l[NT], z[NT];                 // of heads 2t, 2t + 1: -m, infinite without a key; l and z: this lane's share
};

// Streams tiles [first, first + count) of a segment.
template <int D, int kBits, int NT>
__device__ __forceinline__ void stream_tiles(const DecodeArgs& a, const Cache& c, const Segment& s, int count, uint8_t* ring,
                                             uint32_t bars, volatile uint32_t* there, uint32_t& phases, int lane,
                                             Piece<D, kBits, NT>& pc) {
  using S = Shape<D, kBits, NT>;
  constexpr int MG = 1;                          // groups of 16 keys at a time
  constexpr int DG = D / 8;                      // values of a lane's stretch of the output
  const int g = lane >> 2, t = lane & 3;
  const int kv = s.unit / a.chunks, chunk = s.unit - kv * a.chunks;
  const int rows = min(a.rows, a.group - chunk * a.rows);
  const uint32_t ring_at = smem_addr(ring);
  const int32_t* table = a.table + int64_t(s.b) * a.max_pages;
  const int pgroup = kBits == 4 ? kv * D / kGroup : 0;

  // ---- loads: a lane copies one run of rows, the part of a tile that lies in one page ----
  const int run = min(c.page_size, S::kKeys);
  const int run_shift = min(c.page_shift, S::kKeys == 32 ? 5 : 4);
  constexpr int kArrays = kBits == 4 ? 4 : 2;    // keys, values, their steps and zero points
  const int copies = kArrays * (S::kKeys >> run_shift);
  auto page_of = [&](int tile, int copy) -> int {                    // of a copy's run; -1 if there is none
    const int64_t key = int64_t(tile) * S::kKeys + (int64_t(copy / kArrays) << run_shift);
    if (copy >= copies || key >= s.length) return -1;
    const int p = __ldg(table + (key >> c.page_shift));
    if (p >= 0 && p < c.pages) return p;
    atomicCAS(&g_decode_status, 0, int(kDecodeRange));
    return -1;
  };
  // this lane's copy of a tile that is all there
  const int my_array = lane % kArrays, my_first = (lane / kArrays) << run_shift;
  const uint32_t my_bytes = my_array < 2 ? S::kRowBytes : 8;         // a key
  const uint8_t* my_src = my_array == 0 ? static_cast<const uint8_t*>(c.k) : static_cast<const uint8_t*>(c.v);
  uint32_t my_dst = ring_at + (my_array * S::kKeys + my_first) * S::kRowBytes;
  int my_heads = c.kv_heads, my_head = kv;
  if (my_array >= 2) {
    my_src = reinterpret_cast<const uint8_t*>(my_array == 2 ? c.k_params : c.v_params);
    my_dst = ring_at + 2 * S::kKeys * S::kRowBytes + ((my_array - 2) * S::kKeys + my_first) * 8;
    my_heads = c.groups;
    my_head = pgroup;
  }
  my_src += (int64_t(my_head) << c.page_shift) * my_bytes;
  const uint32_t my_page = (uint32_t(my_heads) << c.page_shift) * my_bytes;      // below 2^31 (checked)
  const uint32_t my_size = my_bytes << run_shift;
  const bool one_each = copies <= 32 && (kBits == 16 || run > 1);

  auto issue = [&](int tile, int page, int stage) {
    const uint32_t at = ring_at + stage * S::kStageBytes, bar = bars + 8 * stage;
    if (one_each && uint32_t(tile + 1) * S::kKeys <= uint32_t(s.length) && __all_sync(0xffffffffu, page >= 0 || lane >= copies)) {
      if (lane == 0) {
        there[stage] = S::kKeys == 32 ? 0xFFFFFFFFu : 0xFFFFu;
        bar_expect(bar, S::kStageBytes);
      }
      __syncwarp();
      if (lane < copies) {
        const uint32_t offset = uint32_t(tile * S::kKeys + my_first) & uint32_t(c.page_size - 1);
        copy_rows(my_dst + stage * S::kStageBytes, my_src + uint64_t(uint32_t(page)) * my_page + offset * my_bytes, my_size, bar);
      }
      return;
    }
    uint32_t keys = 0, bytes = 0;
    for (int copy = lane; copy < copies; copy += 32) {
      if (copy >= 32) page = page_of(tile, copy);
      const int array = copy % kArrays, first = (copy / kArrays) << run_shift;
      const int n = page < 0 ? 0 : min(run, s.length - tile * S::kKeys - first);
      if (array == 0) keys |= n == 0 ? 0u : (0xFFFFFFFFu >> (32 - n)) << first;
      if (array < 2) bytes += n * S::kRowBytes;
      else if (run > 1) bytes += (n + 1) / 2 * 16;                   // a copy is a multiple of 16 bytes
    }
    keys = __reduce_or_sync(0xffffffffu, keys);
    bytes = __reduce_add_sync(0xffffffffu, bytes);
    if (lane == 0) {
      there[stage] = keys;
      bar_expect(bar, bytes);
    }
    __syncwarp();
    if (copies > 32) page = page_of(tile, lane);
    for (int copy = lane; copy < copies; copy += 32) {
      if (copy >= 32) page = page_of(tile, copy);
      const int array = copy % kArrays, first = (copy / kArrays) << run_shift;
      const int n = page < 0 ? 0 : min(run, s.length - tile * S::kKeys - first);
      if (n == 0) continue;
      const int offset = (tile * S::kKeys + first) & (c.page_size - 1);
      const uint8_t* src;
      uint32_t dst, size;
      if (array < 2) {
        src = static_cast<const uint8_t*>(array ? c.v : c.k) + head_row(c, page, kv, offset) * S::kRowBytes;
        dst = at + (array * S::kKeys + first) * S::kRowBytes;
        size = n * S::kRowBytes;
      } else {
        src = reinterpret_cast<const uint8_t*>((array == 2 ? c.k_params : c.v_params) + param_row(c, page, pgroup, offset));
        dst = at + 2 * S::kKeys * S::kRowBytes + ((array - 2) * S::kKeys + first) * 8;
        size = (n + 1) / 2 * 16;
        if (run == 1) {                          // pages of one token: 8 bytes
          const float2 x = *reinterpret_cast<const float2*>(src);
          asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(dst), "f"(x.x), "f"(x.y) : "memory");
          continue;
        }
      }
      copy_rows(dst, src, size, bar);
    }
    __syncwarp();                                // those stores are seen by the other lanes: the barrier waits for copies only
  };
  for (int i = 0; i < S::kStages && i < count; ++i) issue(s.tile + i, page_of(s.tile + i, lane), i);
  int page = S::kStages < count ? page_of(s.tile + S::kStages, lane) : -1;

  // ---- queries: the second operand of K Q^T, heads in columns; column g of group n is head 8 n + g ----
  uint32_t q[NT][D / 16][2];
  f32x2 qsum[NT];                                // of heads 2t, 2t + 1
  float qodd[NT][2];                             // where the sum of q.c starts: 8 sum(q) - 72 sum over odd values
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int h = 8 * n + g;
    const __half* src = a.q + int64_t(s.b) * a.ldq + (int64_t(kv) * a.group + chunk * a.rows + h) * D;
    float sum = 0.0f, odd = 0.0f;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {           // 8 values: two steps of 16
      uint4 x = make_uint4(0, 0, 0, 0);
      const int at = kBits == 4 ? t * (D / 4) + 8 * w : 32 * w + 8 * t;
      if (h < rows) x = __ldg(reinterpret_cast<const uint4*>(src + at));
      if (kBits == 4) {                          // the order that codes_to_half gives
        q[n][2 * w][0] = prmt(x.x, x.z, 0x5410);
        q[n][2 * w][1] = prmt(x.x, x.z, 0x7632);
        q[n][2 * w + 1][0] = prmt(x.y, x.w, 0x5410);
        q[n][2 * w + 1][1] = prmt(x.y, x.w, 0x7632);
        const uint32_t* u = reinterpret_cast<const uint32_t*>(&x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(u + i));
          sum += f.x + f.y;
          odd += f.y;
        }
      } else {
        q[n][2 * w][0] = x.x;
        q[n][2 * w][1] = x.y;
        q[n][2 * w + 1][0] = x.z;
        q[n][2 * w + 1][1] = x.w;
      }
    }
    if (kBits == 4) {
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      const float s0 = __shfl_sync(0xffffffffu, sum, 8 * t), s1 = __shfl_sync(0xffffffffu, sum, 8 * t + 4);
      qsum[n] = pack2(s0, s1);
      odd += __shfl_xor_sync(0xffffffffu, odd, 1);
      odd += __shfl_xor_sync(0xffffffffu, odd, 2);
      qodd[n][0] = fmaf(-72.0f, __shfl_sync(0xffffffffu, odd, 8 * t), 8.0f * s0);
      qodd[n][1] = fmaf(-72.0f, __shfl_sync(0xffffffffu, odd, 8 * t + 4), 8.0f * s1);
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    pc.neg_m[n] = pack2(kNoMaximum, kNoMaximum);
    pc.l[n] = pc.z[n] = pack2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) pc.o[i][n][e] = 0.0f;
  }

  const int key_lo = key_of_row(g), key_hi = key_of_row(g + 8);
  constexpr int kParts = S::kKeys / 16;
  float sc2[kParts][NT][4];
  uint32_t pt[MG][NT][2], seen = 0;              // the second operand of V^T P^T; keys of this tile
  bool full = false;
  auto arrived = [&](int stage) -> bool {
    if (!bar_wait(bars + 8 * stage, (phases >> stage) & 1)) return false;
    seen = there[stage];
    full = seen == (S::kKeys == 32 ? 0xFFFFFFFFu : 0xFFFFu);
    const uint32_t none = phases & kNoKey;
    phases = (phases ^ (1u << stage)) & ~kNoKey;
    if (!full && seen == 0) phases |= none;
    if (kBits == 16 && !full) {                  // 0 * NaN is NaN: values of keys that are not there are zeroed
      for (int x = lane; x < S::kKeys * (S::kRowBytes / 16); x += 32)
        if (((seen >> (x / (S::kRowBytes / 16))) & 1) == 0)
          reinterpret_cast<uint4*>(ring + stage * S::kStageBytes + S::kKeys * S::kRowBytes)[x] = make_uint4(0, 0, 0, 0);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
    }
    return true;
  };
  auto scores = [&](int stage, int part) {
    const uint8_t* kt = ring + stage * S::kStageBytes + part * 16 * S::kRowBytes;
    // ---- S^T = K Q^T ----
    float sa[NT][4];
#pragma unroll
    for (int mg = 0; mg < MG; ++mg) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sa[n][e] = kBits == 4 ? qodd[n][e & 1] : 0.0f;
        }
      const uint8_t* lo = kt + (16 * mg + key_lo) * S::kRowBytes;
      const uint8_t* hi = kt + (16 * mg + key_hi) * S::kRowBytes;
      if (kBits == 4) {
        uint32_t wl[D / 32], wh[D / 32];
        if (D == 128) {
          *reinterpret_cast<uint4*>(wl) = *reinterpret_cast<const uint4*>(lo + t * 16);
          *reinterpret_cast<uint4*>(wh) = *reinterpret_cast<const uint4*>(hi + t * 16);
        } else {
          *reinterpret_cast<uint2*>(wl) = *reinterpret_cast<const uint2*>(lo + t * 8);
          *reinterpret_cast<uint2*>(wh) = *reinterpret_cast<const uint2*>(hi + t * 8);
        }
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
          uint32_t x[4], y[4];
          key_codes_to_half(wl[w], x);
          key_codes_to_half(wh[w], y);
          const uint32_t a0[4] = {x[0], y[0], x[1], y[1]}, a1[4] = {x[2], y[2], x[3], y[3]};
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma16816(sa[n], a0, q[n][2 * w][0], q[n][2 * w][1]);
            mma16816(sa[n], a1, q[n][2 * w + 1][0], q[n][2 * w + 1][1]);
          }
        }
      } else {
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
          const uint4 x = *reinterpret_cast<const uint4*>(lo + w * 64 + t * 16);
          const uint4 y = *reinterpret_cast<const uint4*>(hi + w * 64 + t * 16);
          const uint32_t a0[4] = {x.x, y.x, x.y, y.y}, a1[4] = {x.z, y.z, x.w, y.w};
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma16816(sa[n], a0, q[n][2 * w][0], q[n][2 * w][1]);
            mma16816(sa[n], a1, q[n][2 * w + 1][0], q[n][2 * w + 1][1]);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc2[part][n][e] = sa[n][e];
    }
  };
  auto weigh = [&](int stage, int part) {
    const float2* kp = reinterpret_cast<const float2*>(ring + stage * S::kStageBytes + 2 * S::kKeys * S::kRowBytes) + 16 * part;
    const float2* vp = kp + S::kKeys;
    const uint32_t seen16 = seen >> (16 * part);
    // ---- weights ----
    // x = (q.c - z sum(q)) s_k c, y = x - m, w = 2^y s_v.  Heads 2t and 2t + 1 go through packed arithmetic.
    float ks[MG][2], kz[MG][2], sv[MG][2], zv[MG][2];
    f32x2 y[MG][2][NT];
#pragma unroll
    for (int mg = 0; mg < MG; ++mg) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int key = 16 * mg + (r ? key_hi : key_lo);
        ks[mg][r] = a.c;
        kz[mg][r] = 0.0f;
        sv[mg][r] = 1.0f;
        zv[mg][r] = 0.0f;
        if (kBits == 4) {
          const float2 k2 = kp[key], v2 = vp[key];
          ks[mg][r] = k2.x * a.c;
          kz[mg][r] = -k2.y * ks[mg][r];         // the 8 that the codes lack is in where their sum starts
          sv[mg][r] = v2.x;
          zv[mg][r] = v2.y - 8.0f;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          f32x2 u = pc.neg_m[n];
          if (kBits == 4) u = fma2(pack2(kz[mg][r], kz[mg][r]), qsum[n], u);
          y[mg][r][n] = fma2(pack2(sc2[part][n][2 * r], sc2[part][n][2 * r + 1]), pack2(ks[mg][r], ks[mg][r]), u);
        }
      }
    }
    if (!full) {                                 // keys that are not there: no weight, whatever their places hold
#pragma unroll
      for (int mg = 0; mg < MG; ++mg) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if ((seen16 >> (16 * mg + (r ? key_hi : key_lo))) & 1) continue;
          sv[mg][r] = 1.0f;
          zv[mg][r] = 0.0f;
#pragma unroll
          for (int n = 0; n < NT; ++n) y[mg][r][n] = pack2(-INFINITY, -INFINITY);
        }
      }
    }
    f32x2 p2[MG][2][NT], w2[MG][2][NT];
    float high = 0.0f;
    auto weights = [&]() {
#pragma unroll
      for (int mg = 0; mg < MG; ++mg) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float y0, y1, w0, w1;
            unpack2(y[mg][r][n], y0, y1);
            p2[mg][r][n] = pack2(exp2_fast(y0), exp2_fast(y1));
            w2[mg][r][n] = kBits == 4 ? mul2(p2[mg][r][n], pack2(sv[mg][r], sv[mg][r])) : p2[mg][r][n];
            unpack2(w2[mg][r][n], w0, w1);
            high = fmaxf(high, fmaxf(w0, w1));
          }
        }
      }
    };
    weights();
    if (__any_sync(0xffffffffu, high > 32768.0f)) {
      if (kBits == 4) {                          // rows of zeros among the values: the four lanes of a key look at a quarter each
        bool flat[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) flat[r] = sv[0][r] == 1.0f && zv[0][r] == -8.0f;
        if (__any_sync(0xffffffffu, flat[0] || flat[1])) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const uint8_t* row = ring + stage * S::kStageBytes + (S::kKeys + 16 * part + (r ? key_hi : key_lo)) * S::kRowBytes;
            uint32_t codes = 0;
#pragma unroll
            for (int i = 0; i < S::kRowBytes / 16; ++i) codes |= reinterpret_cast<const uint32_t*>(row)[t * (S::kRowBytes / 16) + i];
            codes |= __shfl_xor_sync(0xffffffffu, codes, 1);
            codes |= __shfl_xor_sync(0xffffffffu, codes, 2);
            if (flat[r] && codes == 0) sv[0][r] = kStepOfZeros;
          }
        }
      }
      // a new m, from x itself: y has lost its places where m was far off
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float m[2], to[2], keep[2], qs[2] = {0.0f, 0.0f};
        unpack2(pc.neg_m[n], m[0], m[1]);
        if (kBits == 4) unpack2(qsum[n], qs[0], qs[1]);
        to[0] = -m[0];
        to[1] = -m[1];
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
          for (int mg = 0; mg < MG; ++mg) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const bool live = (seen16 >> (16 * mg + (r ? key_hi : key_lo))) & 1;
              const float lead = kBits == 4 ? log2_fast(sv[mg][r]) : 0.0f;
              float x[2];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                x[e] = live ? fmaf(sc2[part][n][2 * r + e], ks[mg][r], kz[mg][r] * qs[e]) : -INFINITY;
                if (pass == 0) to[e] = fmaxf(to[e], x[e] + lead - 7.0f);
              }
              if (pass == 1) y[mg][r][n] = pack2(x[0] - to[0], x[1] - to[1]);
            }
          }
          if (pass == 0) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
              for (int o = 4; o < 32; o <<= 1) to[e] = fmaxf(to[e], __shfl_xor_sync(0xffffffffu, to[e], o));
              keep[e] = exp2_fast(-m[e] - to[e]);
            }
          }
        }
        pc.neg_m[n] = pack2(-to[0], -to[1]);
        const f32x2 k2 = pack2(keep[0], keep[1]);
        pc.l[n] = mul2(pc.l[n], k2);
        pc.z[n] = mul2(pc.z[n], k2);
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) pc.o[x][n][e] *= keep[e & 1];
      }
      weights();
    }
#pragma unroll
    for (int mg = 0; mg < MG; ++mg) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          pc.l[n] = add2(pc.l[n], p2[mg][r][n]);
          float w0, w1;
          unpack2(w2[mg][r][n], w0, w1);
          const __half2 h = __floats2half2_rn(w0, w1);
          const uint32_t bits = *reinterpret_cast<const uint32_t*>(&h);
          if (kBits == 4) pc.z[n] = fma2(half2_to_f32x2(bits), pack2(zv[mg][r], zv[mg][r]), pc.z[n]);
          pt[mg][n][r] = transposed(bits);
        }
      }
    }
  };
  auto values = [&](int stage, int part) {
    const uint8_t* vt = ring + stage * S::kStageBytes + (S::kKeys + part * 16) * S::kRowBytes;
    // ---- O^T += V^T P^T ----
#pragma unroll
    for (int mg = 0; mg < MG; ++mg) {
      const uint8_t* v0 = vt + (16 * mg + t) * S::kRowBytes;
      const uint8_t* v1 = vt + (16 * mg + 4 + (t ^ 1)) * S::kRowBytes;
      const uint8_t* v2 = v0 + 8 * S::kRowBytes;
      const uint8_t* v3 = v1 + 8 * S::kRowBytes;
      if (kBits == 4) {
        uint32_t w0[2], w1[2], w2[2], w3[2];
        if (D == 128) {
          *reinterpret_cast<uint2*>(w0) = *reinterpret_cast<const uint2*>(v0 + g * 8);
          *reinterpret_cast<uint2*>(w1) = *reinterpret_cast<const uint2*>(v1 + g * 8);
          *reinterpret_cast<uint2*>(w2) = *reinterpret_cast<const uint2*>(v2 + g * 8);
          *reinterpret_cast<uint2*>(w3) = *reinterpret_cast<const uint2*>(v3 + g * 8);
        } else {
          w0[0] = *reinterpret_cast<const uint32_t*>(v0 + g * 4);
          w1[0] = *reinterpret_cast<const uint32_t*>(v1 + g * 4);
          w2[0] = *reinterpret_cast<const uint32_t*>(v2 + g * 4);
          w3[0] = *reinterpret_cast<const uint32_t*>(v3 + g * 4);
        }
#pragma unroll
        for (int w = 0; w < DG / 8; ++w) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {          // codes 0-3, 4-7 of the word
            const uint32_t sel = half ? 0x7632u : 0x5410u;
            uint32_t x[4], y[4];
            // two keys' four codes side by side: nibble k of the low and of the high half
            codes_to_half(prmt(w0[w], w1[w], sel), x);
            codes_to_half(prmt(w2[w], w3[w], sel), y);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t av[4] = {x[2 * e], x[2 * e + 1], y[2 * e], y[2 * e + 1]};
#pragma unroll
              for (int n = 0; n < NT; ++n) mma16816(pc.o[4 * w + 2 * half + e][n], av, pt[mg][n][0], pt[mg][n][1]);
            }
          }
        }
      } else {
#pragma unroll
        for (int w = 0; w < DG / 8; ++w) {
          const uint4 x0 = *reinterpret_cast<const uint4*>(v0 + g * (2 * DG) + w * 16);
          const uint4 x1 = *reinterpret_cast<const uint4*>(v1 + g * (2 * DG) + w * 16);
          const uint4 x2 = *reinterpret_cast<const uint4*>(v2 + g * (2 * DG) + w * 16);
          const uint4 x3 = *reinterpret_cast<const uint4*>(v3 + g * (2 * DG) + w * 16);
          const uint32_t* u0 = reinterpret_cast<const uint32_t*>(&x0);
          const uint32_t* u1 = reinterpret_cast<const uint32_t*>(&x1);
          const uint32_t* u2 = reinterpret_cast<const uint32_t*>(&x2);
          const uint32_t* u3 = reinterpret_cast<const uint32_t*>(&x3);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t av[4] = {prmt(u0[e], u1[e], 0x5410), prmt(u0[e], u1[e], 0x7632), prmt(u2[e], u3[e], 0x5410),
                                    prmt(u2[e], u3[e], 0x7632)};
#pragma unroll
            for (int n = 0; n < NT; ++n) mma16816(pc.o[4 * w + e][n], av, pt[mg][n][0], pt[mg][n][1]);
          }
        }
      }
    }
  };

  phases |= kNoKey;
  int stage = 0, i = 0;
  for (; i < count; ++i) {
    if (!arrived(stage)) break;
#pragma unroll
    for (int part = 0; part < kParts; ++part) scores(stage, part);
#pragma unroll
    for (int part = 0; part < kParts; ++part) {
      weigh(stage, part);
      values(stage, part);
    }
    __syncwarp();
    if (i + S::kStages < count) {
      issue(s.tile + i + S::kStages, page, stage);
      page = i + S::kStages + 1 < count ? page_of(s.tile + i + S::kStages + 1, lane) : -1;
    }
    stage = stage + 1 == S::kStages ? 0 : stage + 1;
  }
  __syncwarp();
  if (i < count) {                               // a wait ran out: copies under way have time to land
    if (lane == 0) atomicCAS(&g_decode_status, 0, int(kDecodeWait));
    for (int left = min(S::kStages, count - i); left > 0; --left) {
      const unsigned long long t0 = now_ns();
      while (!bar_try(bars + 8 * stage, (phases >> stage) & 1) && now_ns() - t0 < kDecodeDrainNs) {}
      stage = stage + 1 == S::kStages ? 0 : stage + 1;
    }
    __syncwarp();
    phases = kGaveUp;
  }
  // the lanes' shares of the sums; zero points out of the output
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float l[2], z[2];
    unpack2(pc.l[n], l[0], l[1]);
    unpack2(pc.z[n], z[0], z[1]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        l[e] += __shfl_xor_sync(0xffffffffu, l[e], o);
        if (kBits == 4) z[e] += __shfl_xor_sync(0xffffffffu, z[e], o);
      }
      if (kBits == 4) {
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
          pc.o[x][n][e] -= z[e];
          pc.o[x][n][2 + e] -= z[e];
        }
      }
    }
    pc.l[n] = pack2(l[0], l[1]);
  }
  // told from a piece whose scores are all -infinity
  if ((phases & kNoKey) != 0) {
#pragma unroll
    for (int n = 0; n < NT; ++n) pc.neg_m[n] = pack2(INFINITY, INFINITY);
  }
}

template <int D, int kBits, int NT>
__global__ void __launch_bounds__(kDecodeThreads, Shape<D, kBits, NT>::kCtas)
attn_decode_kernel(const DecodeArgs a, const Cache c) {
  using S = Shape<D, kBits, NT>;
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int record = a.rows * (D + 2);                      // floats: output, reference, sum
  const int stride = (record + 3) / 4 * 4;                  // of the records in the workspace
  uint8_t* ring = smem + warp * S::kWarpBytes;
  float* heads_of = reinterpret_cast<float*>(smem + kWarps * S::kWarpBytes);    // [warp][record]: pieces that began in an earlier warp
  __shared__ int s_sums[kDecodeThreads + 1];
  __shared__ int s_scan[kWarps], s_most[kWarps];
  __shared__ int s_seg[16], s_flag[16];     // the records' segments; bit 0: its first tile, bit 1: its last, bit 2: the record is not there
  __shared__ __align__(8) unsigned long long s_bars[kWarps][S::kStages];   // a stage's copies
  __shared__ uint32_t s_there[kWarps][S::kStages];          // and the keys that they bring
  __shared__ float s_total[8 * NT];
  __shared__ int s_missing;                                 // 1 + k: a CTA has not got its piece of pending segment k

  // ---- the line of tiles: the sequences' tile counts, added up by the whole CTA ----
  const int per = (a.batch + kDecodeThreads - 1) / kDecodeThreads;
  // The start of a segment (queries, an empty ring) costs a warp about as much as a tile, and counts as one: tile 0 of
  // the line's tiles of a segment is no work, tile i + 1 the i-th of its keys.
  auto tiles_of = [&](int b) {
    const int n = int((uint32_t(clamped_length(a, c, b)) + S::kKeys - 1) / S::kKeys);      // a length may be just below 2^31
    return n == 0 ? 0 : n + 1;
  };
  int mine = 0, most = 0;
  for (int b = min(a.batch, tid * per); b < min(a.batch, tid * per + per); ++b) {
    const int n = tiles_of(b);
    mine += n;
    most = max(most, n);
    if (blockIdx.x == 0) {
      const int len = a.lengths[b];
      if (len < 0 || len > (a.max_pages << c.page_shift)) atomicCAS(&g_decode_status, 0, int(kDecodeRange));
    }
    if (n == 0 && b % gridDim.x == blockIdx.x) {            // an empty sequence: zeros
      for (int i = 0; i < a.units / a.chunks * a.group * D / 8; ++i)
        reinterpret_cast<uint4*>(a.y + int64_t(b) * a.ldy)[i] = make_uint4(0, 0, 0, 0);
    }
  }
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
    most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
  }
  if (lane == 31) s_scan[warp] = incl;
  if (lane == 0) s_most[warp] = most;
  if (tid < 16) s_seg[tid] = -1;
  const uint32_t bars = smem_addr(&s_bars[warp][0]);
  if (lane < S::kStages) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + 8 * lane) : "memory");
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  uint32_t phases = g_decode_wait_limit_ns < kAtOnceNs ? kGaveUp : 0;     // bit i: parity of stage i's next use
  __syncthreads();
  for (int i = 0; i < kWarps; ++i) {
    if (i < warp) incl += s_scan[i];
    most = max(most, s_most[i]);
  }
  s_sums[tid + 1] = incl;
  if (tid == 0) s_sums[0] = 0;
  __syncthreads();
  const int all = s_sums[kDecodeThreads] * a.units;         // tiles in the line: below 2^31 (checked)
  const int segments = a.batch * a.units;
  // Short sequences: a CTA per segment, so that nothing has to meet in the workspace.  Else equal stretches.  This / the other, us, at
  // equal lengths, 32 + 8 heads of 128 in 4 bits: 1 sequence of 64 tokens 7.8 / 12.3, 512 10.1 / 13.4, 1024 13.3 / 13.6, 1200
  // 15.1 / 13.1, 4096 34 / 15; 32 sequences (256 segments, nearly a CTA each anyway) 512 12.8 / 18.3, 1024 17.9 / 23.9, 2048
  // 28.0 / 32.2, 4096 47.4 / 48.1, which this rule leaves to the other.  fp16, 32 + 32 heads, 1 sequence: 64 6.4 / 11.3, 512 11.5 / 12.1,
  // 768 13.8 / 13.2.
  const bool whole = segments <= int(gridDim.x) && most <= 4 * kWarps + 1;
  const int ctas = whole ? segments : min(int(gridDim.x), (all + kWarps - 1) / kWarps);
  if (int(blockIdx.x) >= ctas) return;

  auto start_of_sequence = [&](int b) -> int {              // tiles per unit before sequence b
    const int i = b / per;
    int at = s_sums[i];
    for (int x = i * per; x < b; ++x) at += tiles_of(x);
    return at;
  };
  // CTA i's stretch starts at tile i * share + min(i, extra)
  const int share = all / ctas, extra = all - share * ctas;
  auto start_of_cta = [&](int i) -> int { return i * share + min(i, extra); };
  auto cta_of = [&](int tile) -> int {
    const int bound = extra * (share + 1);
    return tile < bound ? tile / (share + 1) : extra + (tile - bound) / share;
  };
  int begin, end;                                           // this warp's stretch
  if (whole) {
    const int b = blockIdx.x / a.units, n = tiles_of(b);
    const int at = start_of_sequence(b) * a.units + (blockIdx.x - b * a.units) * n;
    if (n == 0) return;
    begin = at + 1 + (n - 1) * warp / kWarps;
    end = at + 1 + (n - 1) * (warp + 1) / kWarps;
  } else {
    begin = start_of_cta(blockIdx.x);
    const int n = share + (int(blockIdx.x) < extra ? 1 : 0), each = n / kWarps, more = n % kWarps;
    begin += warp * each + min(warp, more);
    end = begin + each + (warp < more ? 1 : 0);
  }

  if ((phases & kGaveUp) != 0 && lane == 0) atomicCAS(&g_decode_status, 0, int(kDecodeWait));
  if (begin < end) {
    // the segment of tile `begin`: sequence b with start(b) * units <= begin < start(b + 1) * units
    Segment s;
    int lo = 0, hi = kDecodeThreads;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (s_sums[mid] * a.units <= begin) lo = mid; else hi = mid;
    }
    int at = s_sums[lo] * a.units;
    s.b = lo * per;
    s.tiles = tiles_of(s.b);
    while (at + s.tiles * a.units <= begin) {
      at += s.tiles * a.units;
      s.tiles = tiles_of(++s.b);
    }
    s.unit = (begin - at) / s.tiles;
    s.tile = (begin - at) - s.unit * s.tiles;
    while (true) {
      s.length = clamped_length(a, c, s.b);
      const int place = s.tile, steps = min(s.tiles - place, end - begin);
      const bool first = place <= 1, last = place + steps == s.tiles;
      const int count = place == 0 ? steps - 1 : steps;
      s.tile = place == 0 ? 0 : place - 1;
      if (count > 0) {
      Piece<D, kBits, NT> pc;
      if ((phases & kGaveUp) == 0) stream_tiles<D, kBits, NT>(a, c, s, count, ring, bars, s_there[warp], phases, lane, pc);
      const bool lost = (phases & kGaveUp) != 0;            // this piece, as all that follow in this warp
      const int g = lane >> 2, t = lane & 3;
      const int kv = s.unit / a.chunks, chunk = s.unit - kv * a.chunks;
      const int rows = min(a.rows, a.group - chunk * a.rows);
      float pl[NT][2], pm[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        unpack2(pc.l[n], pl[n][0], pl[n][1]);
        unpack2(pc.neg_m[n], pm[n][0], pm[n][1]);
      }
      if (first && last) {                                  // the whole segment
        if (!lost) {
        __half* y = a.y + int64_t(s.b) * a.ldy + (int64_t(kv) * a.group + chunk * a.rows) * D + g * (D / 8);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int h = 8 * n + 2 * t + e;
            if (h >= rows) continue;
            const float inv = pm[n][e] == INFINITY ? 0.0f : 1.0f / pl[n][e];      // no token: 0
#pragma unroll
            for (int x = 0; x < D / 64; ++x) {
              uint4 out;
              __half2* o2 = reinterpret_cast<__half2*>(&out);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                o2[i] = __floats2half2_rn(pc.o[4 * x + i][n][e] * inv, pc.o[4 * x + i][n][2 + e] * inv);
              reinterpret_cast<uint4*>(y + h * D)[x] = out;
            }
          }
        }
        }
      } else {
        const int slot = 2 * warp + (first ? 1 : 0);
        float* rec = first ? reinterpret_cast<float*>(ring) : heads_of + warp * record;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int h = 8 * n + 2 * t + e;
            if (h >= rows || lost) continue;
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
              *reinterpret_cast<float2*>(rec + h * D + g * (D / 8) + 2 * i) = make_float2(pc.o[i][n][e], pc.o[i][n][2 + e]);
            if (g == 0) {
              rec[a.rows * D + h] = -pm[n][e];
              rec[a.rows * D + a.rows + h] = pl[n][e];
            }
          }
        }
        if (lane == 0) {
          s_seg[slot] = s.b * a.units + s.unit;
          s_flag[slot] = (first ? 1 : 0) | (last ? 2 : 0) | (lost ? 4 : 0);
        }
      }
      }
      begin += steps;
      if (begin >= end) break;
      s.tile = 0;
      if (++s.unit == a.units) {
        s.unit = 0;
        do s.tiles = tiles_of(++s.b); while (s.tiles == 0);
      }
    }
  }
  __syncthreads();

  // ---- pieces of one segment within the CTA: neighbours in the list of records ----
  auto rec_of = [&](int i) -> float* {
    return (i & 1) ? reinterpret_cast<float*>(smem + (i >> 1) * S::kWarpBytes) : heads_of + (i >> 1) * record;
  };
  int pending[2] = {-1, -1};
  uint32_t missing = 0;                                     // bit k: pending piece k is not there
  {
    // lane i of every warp: record i.  A segment's records find each other by its number.
    const int i = lane & 15, seg = lane < 16 ? s_seg[i] : -1;
    const uint32_t same = __match_any_sync(0xffffffffu, lane < 16 && seg >= 0 ? seg : ~lane) ;
    const uint32_t leads = __ballot_sync(0xffffffffu, seg >= 0 && (same & ((1u << lane) - 1u)) == 0);
    const uint32_t firsts = __ballot_sync(0xffffffffu, seg >= 0 && (s_flag[i] & 1)), lasts = __ballot_sync(0xffffffffu, seg >= 0 && (s_flag[i] & 2));
    const uint32_t losts = __ballot_sync(0xffffffffu, seg >= 0 && (s_flag[i] & 4));
    int task = 0;                                           // (segment, head), a warp each
    for (uint32_t left = leads; left != 0; left &= left - 1) {
      const int lead = __ffs(left) - 1, sg = __shfl_sync(0xffffffffu, seg, lead);
      const uint32_t mask = __shfl_sync(0xffffffffu, same, lead);
      const bool starts = (firsts & mask) != 0, ends = (lasts & mask) != 0;
      const bool lost = (losts & mask) != 0;
      if (!(starts && ends)) {
        pending[starts ? 1 : 0] = sg;
        missing |= lost ? (starts ? 2u : 1u) : 0u;
      }
      if (lost) continue;
      const int b = sg / a.units, unit = sg - b * a.units;
      const int kv = unit / a.chunks, chunk = unit - kv * a.chunks;
      const int rows = min(a.rows, a.group - chunk * a.rows);
      for (int h = 0; h < rows; ++h, ++task) {
        if (task % kWarps != warp) continue;
        const bool mine = (mask >> lane) & 1;
        const float m = mine ? rec_of(i)[a.rows * D + h] : -INFINITY;
        float l = mine ? rec_of(i)[a.rows * D + a.rows + h] : 0.0f, top = m;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float f = mine ? (top == -INFINITY ? 1.0f : exp2_fast(m - top)) : 0.0f;
        l *= f;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        l = __shfl_sync(0xffffffffu, l, 0);
        float o[D / 32] = {};
        for (uint32_t x = mask; x != 0; x &= x - 1) {
          const int r = __ffs(x) - 1;
          const float fr = __shfl_sync(0xffffffffu, f, r);
          const float* at = rec_of(r) + h * D + lane * 2;
#pragma unroll
          for (int k = 0; k < D / 64; ++k) {
            const float2 v = *reinterpret_cast<const float2*>(at + 64 * k);
            o[2 * k] = fmaf(v.x, fr, o[2 * k]);
            o[2 * k + 1] = fmaf(v.y, fr, o[2 * k + 1]);
          }
        }
        if (starts && ends) {
          __half* y = a.y + int64_t(b) * a.ldy + (int64_t(kv) * a.group + chunk * a.rows + h) * D + lane * 2;
          const float inv = __shfl_sync(0xffffffffu, top, 0) == -INFINITY ? 0.0f : 1.0f / l;      // no token: 0
#pragma unroll
          for (int k = 0; k < D / 64; ++k)
            *reinterpret_cast<__half2*>(y + 64 * k) = __floats2half2_rn(o[2 * k] * inv, o[2 * k + 1] * inv);
        } else {
          float* out = a.records + (int64_t(blockIdx.x) * 2 + (starts ? 1 : 0)) * stride;
#pragma unroll
          for (int k = 0; k < D / 64; ++k)
            *reinterpret_cast<float2*>(out + h * D + lane * 2 + 64 * k) = make_float2(o[2 * k], o[2 * k + 1]);
          if (lane == 0) {
            out[a.rows * D + h] = top;
            out[a.rows * D + a.rows + h] = l;
          }
        }
      }
    }
  }

  // ---- segments that reach over several CTAs: the last of them to arrive adds up ----
  // Each CTA raises a flag of its own per piece and then looks at all of the segment's: at least the last to raise sees them
  // all (sequentially consistent fences).  Of those that do, the one that takes the first piece's flag down adds up; it
  // takes the others down too, so that a replay of the same launch starts anew.  A flag is up when it holds this
  // call's tag, whatever the workspace held before.  A piece that is not there, a wait for it having run out, raises its flag
  // all the same, with the tag's last bit: a flag that stays down would leave the others of its segment up, and a replay of
  // this launch, whose tag is the same, would take them for its own.  Such a segment's flags are taken down and nothing else.
  if (pending[0] < 0 && pending[1] < 0) return;
  __syncthreads();
  if (tid == 0) {
    __threadfence();                                        // the records, all threads', before the flags
    volatile unsigned long long* flags = reinterpret_cast<volatile unsigned long long*>(a.arrived) + blockIdx.x * 2;
    if (pending[0] >= 0) flags[0] = a.tag | (missing & 1);
    if (pending[1] >= 0) flags[1] = a.tag | (missing >> 1);
    s_missing = 0;
    __threadfence();                                        // and the flags before any other is looked at
  }
  float* s_weight = reinterpret_cast<float*>(smem);         // [pieces][rows], over what is done with
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    const int seg = pending[k];
    if (seg < 0) continue;
    const int b = seg / a.units, unit = seg - b * a.units;
    const int kv = unit / a.chunks, chunk = unit - kv * a.chunks;
    const int rows = min(a.rows, a.group - chunk * a.rows);
    __half* y = a.y + int64_t(b) * a.ldy + (int64_t(kv) * a.group + chunk * a.rows) * D;
    const int n = tiles_of(b);
    const int from = start_of_sequence(b) * a.units + unit * n;
    const int c0 = cta_of(from + 1), c1 = cta_of(from + n - 1);
    bool up = true;
    __syncthreads();                                        // this CTA's own flags are up
    for (int i = c0 + tid; i <= c1; i += kDecodeThreads) {
      const unsigned long long flag = reinterpret_cast<volatile unsigned long long*>(a.arrived)[i * 2 + (i == c0 ? 1 : 0)];
      up &= (flag & ~1ull) == a.tag;
      if (flag == (a.tag | 1)) s_missing = 1 + k;
    }
    bool won = __syncthreads_and(up) != 0;
    if (won) {
      bool taken = false;
      if (tid == 0) {
        unsigned long long* flag = a.arrived + c0 * 2 + 1;
        const unsigned long long held = atomicCAS(flag, a.tag, 0ull);
        taken = held == a.tag || (held == (a.tag | 1) && atomicCAS(flag, held, 0ull) == held);
      }
      won = __syncthreads_or(taken) != 0;
    }
    if (won && s_missing != 1 + k) {
      __threadfence();
      auto piece = [&](int i) -> const float* { return a.records + (int64_t(i) * 2 + (i == c0 ? 1 : 0)) * stride; };
      // Everything is asked for at once: the pieces' references and sums, to shared memory, and the first kEarly pieces of this
      // thread's two values.
      const int pieces = c1 - c0 + 1;
      constexpr int kEarly = 8;
      float2 early[kEarly];
      const bool mine = tid * 2 < rows * D;
#pragma unroll
      for (int i = 0; i < kEarly; ++i)
        early[i] = mine && i < pieces ? __ldcg(reinterpret_cast<const float2*>(piece(c0 + i) + tid * 2)) : make_float2(0.0f, 0.0f);
      for (int x = tid; x < pieces * rows; x += kDecodeThreads) {
        const int i = x / rows, h = x - i * rows;
        s_weight[x] = __ldcg(piece(c0 + i) + a.rows * D + h);
        s_weight[pieces * rows + x] = __ldcg(piece(c0 + i) + a.rows * D + a.rows + h);
      }
      __syncthreads();
      for (int h = warp; h < rows; h += kWarps) {           // a warp per head: weights and sum
        float m = -INFINITY, l = 0.0f;
        for (int i = lane; i < pieces; i += 32) m = fmaxf(m, s_weight[i * rows + h]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float ref = m == -INFINITY ? 0.0f : m;
        for (int i = lane; i < pieces; i += 32) {
          const float f = exp2_fast(s_weight[i * rows + h] - ref);
          s_weight[i * rows + h] = f;
          l += s_weight[(pieces + i) * rows + h] * f;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        if (lane == 0) s_total[h] = m == -INFINITY ? INFINITY : l;            // no token: 0
      }
      __syncthreads();
      for (int x = tid * 2; x < rows * D; x += kDecodeThreads * 2) {
        const int h = x / D;
        float o0 = 0.0f, o1 = 0.0f;
        if (x == tid * 2) {
#pragma unroll
          for (int i = 0; i < kEarly; ++i) {
            const float f = i < pieces ? s_weight[i * rows + h] : 0.0f;
            o0 = fmaf(early[i].x, f, o0);
            o1 = fmaf(early[i].y, f, o1);
          }
        }
#pragma unroll 8
        for (int i = x == tid * 2 ? kEarly : 0; i < pieces; ++i) {
          const float2 r = __ldcg(reinterpret_cast<const float2*>(piece(c0 + i) + x));
          const float f = s_weight[i * rows + h];
          o0 = fmaf(r.x, f, o0);
          o1 = fmaf(r.y, f, o1);
        }
        const float inv = 1.0f / s_total[h];
        *reinterpret_cast<__half2*>(y + x) = __floats2half2_rn(o0 * inv, o1 * inv);
      }
      __syncthreads();
    }
    if (won)
      for (int i = c0 + 1 + tid; i <= c1; i += kDecodeThreads) a.arrived[i * 2] = 0;
  }
}

// Test probe: a warp waits, through the kernel's own bounded wait, on a barrier that nobody arrives on.
__global__ void decode_wait_expiry_kernel() {
  __shared__ __align__(8) unsigned long long bar_storage;
  const uint32_t bar = smem_addr(&bar_storage);
  if (threadIdx.x == 0) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncwarp();
  if (!bar_wait(bar, 0) && threadIdx.x == 0) atomicCAS(&g_decode_status, 0, int(kDecodeWait));
}

static void decode_plan(int64_t n_heads, int64_t n_kv, DecodeArgs* a) {
  a->group = int(n_heads / n_kv);
  a->chunks = (a->group + 15) / 16;
  a->rows = (a->group + a->chunks - 1) / a->chunks;
  a->chunks = (a->group + a->rows - 1) / a->rows;
  a->units = int(n_kv) * a->chunks;
}
static int64_t decode_grid() { return int64_t(device_sm_count()) * 2; }

template <int D, int kBits, int NT>
static int launch(const DecodeArgs& a, const Cache& c, cudaStream_t st) {
  using S = Shape<D, kBits, NT>;
  const int grid = device_sm_count() * S::kCtas;
  const int smem = kWarps * (S::kWarpBytes + a.rows * (D + 2) * 4);
  const void* kern = reinterpret_cast<const void*>(&attn_decode_kernel<D, kBits, NT>);
  if (!allow_dynamic_smem(kern, kWarps * (S::kWarpBytes + S::kRecord * 4))) return SMOOTHROT_CUDA_ERROR;
  attn_decode_kernel<D, kBits, NT><<<unsigned(grid), kDecodeThreads, smem, st>>>(a, c);
  count_launch();
  return launch_status();
}

}  // namespace paged
}  // namespace smoothrot

extern "C" {

int smoothrot_decode_status_word(int* out, int clear) {
  return smoothrot::paged::read_status_word(smoothrot::paged::g_decode_status, out, clear);
}

int smoothrot_decode_set_wait_limit_ns(uint64_t ns) {
  const unsigned long long v = ns == 0 ? smoothrot::paged::kDecodeWaitLimitNs : static_cast<unsigned long long>(ns);
  return cudaMemcpyToSymbol(smoothrot::paged::g_decode_wait_limit_ns, &v, sizeof(v)) == cudaSuccess ? SMOOTHROT_OK
                                                                                                   : SMOOTHROT_CUDA_ERROR;
}

int smoothrot_debug_attn_wait_expiry(int code, void* stream) {
  if (code < 36 || code > smoothrot::paged::kDecodeWait) return SMOOTHROT_INVALID_ARG;
  if (code < smoothrot::paged::kDecodeWait) return smoothrot_prefill_wait_expiry(code, stream);
  smoothrot::paged::decode_wait_expiry_kernel<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>();
  smoothrot::count_launch();
  return smoothrot::launch_status();
}

size_t smoothrot_attn_decode_workspace_bytes(int64_t B, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim) {
  using namespace smoothrot::paged;
  if (B <= 0 || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads != 0 || head_dim <= 0) return 0;
  DecodeArgs a;
  decode_plan(n_heads, n_kv_heads, &a);
  return size_t(decode_grid() * 16 + decode_grid() * 2 * ((a.rows * (head_dim + 2) + 3) / 4 * 4) * 4);
}

int smoothrot_attn_decode(const void* Q_f16, int64_t ldq, int64_t B, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                          int bits, int64_t pages, int64_t page_size, const void* k_cache, const void* v_cache,
                          const float* k_params, const float* v_params, const int32_t* block_table, int64_t max_pages,
                          const int32_t* lengths, float scale, void* Y_f16, int64_t ldy, void* workspace,
                          size_t workspace_bytes, void* stream) {
  using namespace smoothrot;
  using namespace smoothrot::paged;
  if (B < 0 || B > 8192 || n_heads <= 0 || n_heads > 65535 || max_pages < 0 || max_pages > INT32_MAX) return SMOOTHROT_INVALID_ARG;
  const int sizes = check_sizes(n_kv_heads, head_dim, bits, pages, page_size);
  if (sizes != SMOOTHROT_OK) return sizes;
  if (n_heads % n_kv_heads != 0 || !(scale == scale)) return SMOOTHROT_INVALID_ARG;
  // a length is an int32, and the tiles of all sequences are counted in one
  if (max_pages * page_size > INT32_MAX || B * (max_pages * page_size / 16 + 2) > INT32_MAX / n_kv_heads / ((n_heads / n_kv_heads + 15) / 16))
    return SMOOTHROT_INVALID_ARG;
  if (B == 0) return SMOOTHROT_OK;
  if (Q_f16 == nullptr || Y_f16 == nullptr || lengths == nullptr || ldq < n_heads * head_dim || ldy < n_heads * head_dim)
    return SMOOTHROT_INVALID_ARG;
  if (max_pages > 0 && block_table == nullptr) return SMOOTHROT_INVALID_ARG;
  if (pages > 0) {
    const int pointers = check_pointers(bits, k_cache, v_cache, k_params, v_params);
    if (pointers != SMOOTHROT_OK) return pointers;
  }
  if (!aligned16(Q_f16) || !aligned16(Y_f16) || ldq % 8 != 0 || ldy % 8 != 0) return SMOOTHROT_BAD_ALIGNMENT;
  if (workspace == nullptr || workspace_bytes < smoothrot_attn_decode_workspace_bytes(B, n_heads, n_kv_heads, head_dim))
    return SMOOTHROT_WORKSPACE_TOO_SMALL;
  if (!aligned16(workspace)) return SMOOTHROT_BAD_ALIGNMENT;
  DecodeArgs a;
  decode_plan(n_heads, n_kv_heads, &a);
  a.q = static_cast<const __half*>(Q_f16); a.ldq = ldq;
  a.table = block_table; a.max_pages = max_pages; a.lengths = lengths;
  a.y = static_cast<__half*>(Y_f16); a.ldy = ldy;
  a.batch = int(B);
  a.c = scale * 1.4426950408889634f;
  a.arrived = static_cast<unsigned long long*>(workspace);
  a.records = reinterpret_cast<float*>(static_cast<char*>(workspace) + decode_grid() * 16);
  // a number that no other call of this process has, and that stray contents of a workspace hardly hold
  static std::atomic<unsigned long long> calls{0x5A17C0DEull};
  a.tag = (calls.fetch_add(1, std::memory_order_relaxed) * 0x9E3779B97F4A7C15ull) << 1;
  const Cache c = make_cache(n_kv_heads, head_dim, bits, pages, page_size, k_cache, v_cache, k_params, v_params);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool wide = a.rows > 8;
  if (head_dim == 128) {
    if (bits == 16) return wide ? launch<128, 16, 2>(a, c, st) : launch<128, 16, 1>(a, c, st);
    return wide ? launch<128, 4, 2>(a, c, st) : launch<128, 4, 1>(a, c, st);
  }
  if (bits == 16) return wide ? launch<64, 16, 2>(a, c, st) : launch<64, 16, 1>(a, c, st);
  return wide ? launch<64, 4, 2>(a, c, st) : launch<64, 4, 1>(a, c, st);
}

}  // extern "C"
