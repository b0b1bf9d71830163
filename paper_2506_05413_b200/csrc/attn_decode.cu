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
// A warp streams its tiles through a ring of its own (cp.async, no barrier with other warps) and computes with the
// warp-level matrix instruction (m16n8k16): the keys of a tile are the 16 rows, the query heads the 8 columns, so a group of
// 4 or 8 heads wastes little, where the tensor-memory instructions would want 128 rows:
//     S^T [keys x heads] = K Q^T,   O^T [values x heads] += V^T P^T
// P leaves S's registers for the second product through movmatrix.  4-bit codes become fp16 whole numbers (exact) in
// registers; step and zero point are applied to the small side:
//     x = (q.c - z sum(q)) s_k,   O = sum w c - sum w z,   w = p s_v
// The weight w is rounded once to fp16, and both sums take the rounded one.  So that w fits fp16 whatever the
// step, the reference m runs over x + log2(s_v); p itself, summed in fp32 for the denominator, may then exceed 1.
// m is raised only where it is exceeded by more than 8, so most tiles need no exchange between lanes.
#include "paged.cuh"

namespace smoothrot {
namespace paged {

__device__ int g_decode_status = 0;

constexpr int kWarps = 8;
constexpr int kDecodeThreads = 32 * kWarps;

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
  unsigned long long* arrived;   // [batch * units]
  float* records;           // [grid][2][rows * D + 2 * rows]
  unsigned long long tag;   // of this call, in the upper 48 bits
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
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(live ? 8 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }

// Codes k and k + 4 of a word (k = 0 .. 3) as two fp16 whole numbers.  0x6400 is 1024 in fp16 with a last place of 1, so
// a code or-ed into it is 1024 + code; four places higher it counts 16 times.
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t (&h)[4]) {
  const uint32_t up = w >> 8;
  uint32_t x[4];
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(x[0]) : "r"(w));
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x64006400, 0xEA;" : "=r"(x[1]) : "r"(w));
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(x[2]) : "r"(up));
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x64006400, 0xEA;" : "=r"(x[3]) : "r"(up));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(h[0]) : "r"(x[0]), "r"(0x64006400u));
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(h[1]) : "r"(x[1]), "r"(0x2C002C00u), "r"(0xD400D400u));   // x / 16 - 64
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(h[2]) : "r"(x[2]), "r"(0x64006400u));
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(h[3]) : "r"(x[3]), "r"(0x2C002C00u), "r"(0xD400D400u));
}

// Key of a tile's 16 that stands in row r of the first product, and so in place r of the second's sum.  A lane's
// four places 2t, 2t+1, 2t+8, 2t+9 of the sum are then rows t, 4 + (t^1), 8 + t, 12 + (t^1): the four lanes of one read
// cover whole rows of values, and two neighbouring rows of keys start in different halves of a 128-byte line.
__device__ __forceinline__ int key_of_row(int r) {
  const int t = (r & 7) >> 1;
  return (r & 8) + ((r & 1) ? 4 + (t ^ 1) : t);
}

template <int D, int kBits, int NT>
struct Piece {                                   // what a warp has of a segment
  float o[D / 16][NT][4];                        // [pairs of values][8 heads][(value 2i, head 2t), (2i, 2t+1), (2i+1, 2t), (2i+1, 2t+1)]
  float m[NT][2], l[NT][2], z[NT][2];            // of heads 2t, 2t + 1; l and z: this lane's share
};

// Streams tiles [first, first + count) of a segment.
template <int D, int kBits, int NT>
__device__ __forceinline__ void stream_tiles(const DecodeArgs& a, const Cache& c, const Segment& s, int count, uint8_t* ring,
                                             int lane, Piece<D, kBits, NT>& pc) {
  using S = Shape<D, kBits, NT>;
  constexpr int MG = S::kKeys / 16;              // groups of 16 keys
  constexpr int DG = D / 8;                      // values of a lane's stretch of the output
  const int g = lane >> 2, t = lane & 3;
  const int kv = s.unit / a.chunks, chunk = s.unit - kv * a.chunks;
  const int rows = min(a.rows, a.group - chunk * a.rows);
  const uint32_t ring_at = smem_addr(ring);
  const int32_t* table = a.table + int64_t(s.b) * a.max_pages;
  const int pgroup = kBits == 4 ? kv * D / kGroup : 0;

  // ---- loads ----
  auto page_of = [&](int tile) -> int {          // the page of key `lane` of a tile; -1 if there is none
    const int64_t key = int64_t(tile) * S::kKeys + lane;
    if (lane >= S::kKeys || key >= s.length) return -1;
    const int p = __ldg(table + (key >> c.page_shift));
    if (p >= 0 && p < c.pages) return p;
    atomicCAS(&g_decode_status, 0, int(kDecodeRange));
    return -1;
  };
  auto issue = [&](int tile, int page, int stage) -> uint32_t {      // returns which keys are there
    const uint32_t there = __ballot_sync(0xffffffffu, page >= 0);
    const uint32_t at = ring_at + stage * S::kStageBytes;
    const int offset = (tile * S::kKeys + lane) & (c.page_size - 1);
    const int64_t row = page >= 0 ? head_row(c, page, kv, offset) : 0;
    constexpr int kChunks = S::kRowBytes / 16;
    constexpr int kPer = 32 / kChunks;           // rows that one instruction covers
#pragma unroll
    for (int i = 0; i < S::kKeys / kPer; ++i) {
      const int key = i * kPer + lane / kChunks, ch = lane % kChunks;
      const int64_t r = __shfl_sync(0xffffffffu, row, key);
      const bool live = (there >> key) & 1;
      const uint32_t dst = at + key * S::kRowBytes + ch * 16;
      const int64_t off = r * S::kRowBytes + ch * 16;
      copy16(dst, static_cast<const uint8_t*>(c.k) + off, live);
      copy16(dst + S::kKeys * S::kRowBytes, static_cast<const uint8_t*>(c.v) + off, live);
    }
    if (kBits == 4) {
      const int64_t r = page >= 0 ? param_row(c, page, pgroup, offset) : 0;
      const uint32_t dst = at + 2 * S::kKeys * S::kRowBytes + lane * 8;
      copy8(dst, c.k_params + r, page >= 0);
      copy8(dst + S::kKeys * 8, c.v_params + r, page >= 0);
    }
    return there;
  };
  uint32_t there[S::kStages];
#pragma unroll
  for (int i = 0; i < S::kStages; ++i) {
    there[i] = 0;
    if (i < count) there[i] = issue(s.tile + i, page_of(s.tile + i), i);
    copy_commit();
  }
  int page = S::kStages < count ? page_of(s.tile + S::kStages) : -1;

  // ---- queries: the second operand of K Q^T, heads in columns; column g of group n is head 8 n + g ----
  uint32_t q[NT][D / 16][2];
  float qsum[NT][2];                             // of heads 2t, 2t + 1
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int h = 8 * n + g;
    const __half* src = a.q + int64_t(s.b) * a.ldq + (int64_t(kv) * a.group + chunk * a.rows + h) * D;
    float sum = 0.0f;
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
      qsum[n][0] = __shfl_sync(0xffffffffu, sum, 8 * t);
      qsum[n][1] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      pc.m[n][e] = -INFINITY;
      pc.l[n][e] = 0.0f;
      pc.z[n][e] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) pc.o[i][n][e] = 0.0f;
  }

  const int key_lo = key_of_row(g), key_hi = key_of_row(g + 8);
  int stage = 0;
  for (int i = 0; i < count; ++i) {
    copy_wait<S::kStages - 1>();
    __syncwarp();
    const uint8_t* kt = ring + stage * S::kStageBytes;
    const uint8_t* vt = kt + S::kKeys * S::kRowBytes;
    const float2* kp = reinterpret_cast<const float2*>(vt + S::kKeys * S::kRowBytes);
    const float2* vp = kp + S::kKeys;
    uint32_t seen = 0;
#pragma unroll
    for (int x = 0; x < S::kStages; ++x) seen = x == stage ? there[x] : seen;

    // ---- S^T = K Q^T ----
    float sc[MG][NT][4];
#pragma unroll
    for (int mg = 0; mg < MG; ++mg) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[mg][n][e] = 0.0f;
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
          codes_to_half(wl[w], x);
          codes_to_half(wh[w], y);
          const uint32_t a0[4] = {x[0], y[0], x[1], y[1]}, a1[4] = {x[2], y[2], x[3], y[3]};
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma16816(sc[mg][n], a0, q[n][2 * w][0], q[n][2 * w][1]);
            mma16816(sc[mg][n], a1, q[n][2 * w + 1][0], q[n][2 * w + 1][1]);
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
            mma16816(sc[mg][n], a0, q[n][2 * w][0], q[n][2 * w][1]);
            mma16816(sc[mg][n], a1, q[n][2 * w + 1][0], q[n][2 * w + 1][1]);
          }
        }
      }
    }

    // ---- weights ----
    float sv[MG][2], zv[MG][2], high[NT][2], lead[MG][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) high[n][0] = high[n][1] = -INFINITY;
#pragma unroll
    for (int mg = 0; mg < MG; ++mg) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int key = 16 * mg + (r ? key_hi : key_lo);
        const bool live = (seen >> key) & 1;
        float2 k2 = make_float2(1.0f, 0.0f);
        sv[mg][r] = 1.0f;
        zv[mg][r] = 0.0f;
        lead[mg][r] = 0.0f;
        if (kBits == 4) {
          k2 = kp[key];
          const float2 v2 = vp[key];
          sv[mg][r] = v2.x;
          zv[mg][r] = v2.y;
          lead[mg][r] = __log2f(v2.x);
        }
        const float ks = k2.x * a.c;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float& x = sc[mg][n][2 * r + e];
            if (kBits == 4) x = fmaf(-k2.y, qsum[n][e], x);
            x *= ks;
            x = live ? x : -INFINITY;
            high[n][e] = fmaxf(high[n][e], x + lead[mg][r]);
          }
        }
      }
    }
    bool raise = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) raise |= high[n][e] > pc.m[n][e] + 8.0f;
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) high[n][e] = fmaxf(high[n][e], __shfl_xor_sync(0xffffffffu, high[n][e], o));
          const float to = fmaxf(pc.m[n][e], high[n][e]);
          const float keep = to == -INFINITY ? 1.0f : exp2_fast(pc.m[n][e] - to);
          pc.m[n][e] = to;
          pc.l[n][e] *= keep;
          pc.z[n][e] *= keep;
#pragma unroll
          for (int x = 0; x < D / 16; ++x) {
            pc.o[x][n][e] *= keep;
            pc.o[x][n][2 + e] *= keep;
          }
        }
      }
    }
    uint32_t pt[MG][NT][2];                      // the second operand of V^T P^T
#pragma unroll
    for (int mg = 0; mg < MG; ++mg) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float w[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float ref = pc.m[n][e] == -INFINITY ? 0.0f : pc.m[n][e];
            const float p = exp2_fast(sc[mg][n][2 * r + e] - ref);
            pc.l[n][e] += p;
            w[e] = kBits == 4 ? p * sv[mg][r] : p;
          }
          const __half2 h = __floats2half2_rn(w[0], w[1]);
          if (kBits == 4) {
            const float2 f = __half22float2(h);
            pc.z[n][0] = fmaf(f.x, zv[mg][r], pc.z[n][0]);
            pc.z[n][1] = fmaf(f.y, zv[mg][r], pc.z[n][1]);
          }
          pt[mg][n][r] = transposed(*reinterpret_cast<const uint32_t*>(&h));
        }
      }
    }

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

    // ---- the stage's next tile ----
    __syncwarp();
    uint32_t next = 0;
    if (i + S::kStages < count) {
      next = issue(s.tile + i + S::kStages, page, stage);
      page = i + S::kStages + 1 < count ? page_of(s.tile + i + S::kStages + 1) : -1;
    }
    copy_commit();
#pragma unroll
    for (int x = 0; x < S::kStages; ++x) there[x] = x == stage ? next : there[x];
    stage = stage + 1 == S::kStages ? 0 : stage + 1;
  }
  copy_wait<0>();
  __syncwarp();
  // the lanes' shares of the sums; zero points out of the output
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        pc.l[n][e] += __shfl_xor_sync(0xffffffffu, pc.l[n][e], o);
        if (kBits == 4) pc.z[n][e] += __shfl_xor_sync(0xffffffffu, pc.z[n][e], o);
      }
      if (kBits == 4) {
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
          pc.o[x][n][e] -= pc.z[n][e];
          pc.o[x][n][2 + e] -= pc.z[n][e];
        }
      }
    }
  }
}

template <int D, int kBits, int NT>
__global__ void __launch_bounds__(kDecodeThreads, Shape<D, kBits, NT>::kCtas)
attn_decode_kernel(const DecodeArgs a, const Cache c) {
  using S = Shape<D, kBits, NT>;
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int record = a.rows * (D + 2);                      // floats: output, reference, sum
  uint8_t* ring = smem + warp * S::kWarpBytes;
  float* heads_of = reinterpret_cast<float*>(smem + kWarps * S::kWarpBytes);    // [warp][record]: pieces that began in an earlier warp
  __shared__ long long s_sums[kDecodeThreads + 1];
  __shared__ int s_scan[kWarps], s_most[kWarps];
  __shared__ int s_seg[2 * kWarps], s_flag[2 * kWarps];     // the records' segments; bit 0: its first tile, bit 1: its last
  __shared__ int s_last;

  // ---- the line of tiles: the sequences' tile counts, added up by the whole CTA ----
  const int per = (a.batch + kDecodeThreads - 1) / kDecodeThreads;
  auto tiles_of = [&](int b) { return (clamped_length(a, c, b) + S::kKeys - 1) / S::kKeys; };
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
  if (tid < 2 * kWarps) s_seg[tid] = -1;
  __syncthreads();
  for (int i = 0; i < kWarps; ++i) {
    if (i < warp) incl += s_scan[i];
    most = max(most, s_most[i]);
  }
  s_sums[tid + 1] = incl;
  if (tid == 0) s_sums[0] = 0;
  __syncthreads();
  const long long all = s_sums[kDecodeThreads] * a.units;   // tiles in the line
  const int segments = a.batch * a.units;
  // Short sequences: a CTA per segment, so that nothing has to meet in the workspace.  Else equal stretches.
  const bool whole = segments <= int(gridDim.x) && most <= 4 * kWarps;
  const int ctas = whole ? segments : int(min((long long)gridDim.x, (all + kWarps - 1) / kWarps));
  if (int(blockIdx.x) >= ctas) return;

  auto start_of_sequence = [&](int b) -> long long {        // tiles per unit before sequence b
    const int i = b / per;
    long long at = s_sums[i];
    for (int x = i * per; x < b; ++x) at += tiles_of(x);
    return at;
  };
  long long begin, end;                                     // this warp's stretch
  if (whole) {
    const int b = blockIdx.x / a.units, n = tiles_of(b);
    const long long at = start_of_sequence(b) * a.units + (long long)(blockIdx.x - b * a.units) * n;
    begin = at + n * warp / kWarps;
    end = at + n * (warp + 1) / kWarps;
  } else {
    const long long w = (long long)blockIdx.x * kWarps + warp, ws = (long long)ctas * kWarps;
    begin = w * all / ws;
    end = (w + 1) * all / ws;
  }

  if (begin < end) {
    // the segment of tile `begin`: sequence b with start(b) * units <= begin < start(b + 1) * units
    Segment s;
    int lo = 0, hi = kDecodeThreads;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (s_sums[mid] * a.units <= begin) lo = mid; else hi = mid;
    }
    long long at = s_sums[lo] * a.units;
    s.b = lo * per;
    s.tiles = tiles_of(s.b);
    while (at + (long long)s.tiles * a.units <= begin) {
      at += (long long)s.tiles * a.units;
      s.tiles = tiles_of(++s.b);
    }
    s.unit = int((begin - at) / s.tiles);
    s.tile = int((begin - at) - (long long)s.unit * s.tiles);
    while (true) {
      s.length = clamped_length(a, c, s.b);
      const int count = int(min((long long)(s.tiles - s.tile), end - begin));
      Piece<D, kBits, NT> pc;
      stream_tiles<D, kBits, NT>(a, c, s, count, ring, lane, pc);
      const int g = lane >> 2, t = lane & 3;
      const int kv = s.unit / a.chunks, chunk = s.unit - kv * a.chunks;
      const int rows = min(a.rows, a.group - chunk * a.rows);
      const bool first = s.tile == 0, last = s.tile + count == s.tiles;
      if (first && last) {                                  // the whole segment
        __half* y = a.y + int64_t(s.b) * a.ldy + (int64_t(kv) * a.group + chunk * a.rows) * D + g * (D / 8);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int h = 8 * n + 2 * t + e;
            if (h >= rows) continue;
            const float inv = 1.0f / pc.l[n][e];
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
      } else {
        const int slot = 2 * warp + (first ? 1 : 0);
        float* rec = first ? reinterpret_cast<float*>(ring) : heads_of + warp * record;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int h = 8 * n + 2 * t + e;
            if (h >= rows) continue;
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
              *reinterpret_cast<float2*>(rec + h * D + g * (D / 8) + 2 * i) = make_float2(pc.o[i][n][e], pc.o[i][n][2 + e]);
            if (g == 0) {
              rec[a.rows * D + h] = pc.m[n][e];
              rec[a.rows * D + a.rows + h] = pc.l[n][e];
            }
          }
        }
        if (lane == 0) {
          s_seg[slot] = s.b * a.units + s.unit;
          s_flag[slot] = (first ? 1 : 0) | (last ? 2 : 0);
        }
      }
      begin += count;
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
  for (int i0 = 0; i0 < 2 * kWarps;) {
    const int seg = s_seg[i0];
    if (seg < 0) {
      ++i0;
      continue;
    }
    int i1 = i0 + 1, flag = s_flag[i0];
    while (i1 < 2 * kWarps && (s_seg[i1] == seg || s_seg[i1] < 0)) {
      if (s_seg[i1] == seg) flag |= s_flag[i1];
      ++i1;
    }
    const int b = seg / a.units, unit = seg - b * a.units;
    const int kv = unit / a.chunks, chunk = unit - kv * a.chunks;
    const int rows = min(a.rows, a.group - chunk * a.rows);
    auto rec_of = [&](int i) -> const float* {
      return (i & 1) ? reinterpret_cast<const float*>(smem + (i >> 1) * S::kWarpBytes) : heads_of + (i >> 1) * record;
    };
    __half* y = a.y + int64_t(b) * a.ldy + (int64_t(kv) * a.group + chunk * a.rows) * D;
    float* out = a.records + (int64_t(blockIdx.x) * 2 + (flag & 1)) * record;
    for (int x = tid; x < rows * D; x += kDecodeThreads) {
      const int h = x / D;
      float m = -INFINITY, l = 0.0f, o = 0.0f;
      for (int i = i0; i < i1; ++i)
        if (s_seg[i] == seg) m = fmaxf(m, rec_of(i)[a.rows * D + h]);
      const float ref = m == -INFINITY ? 0.0f : m;
      for (int i = i0; i < i1; ++i) {
        if (s_seg[i] != seg) continue;
        const float* r = rec_of(i);
        const float f = exp2_fast(r[a.rows * D + h] - ref);
        o += r[x] * f;
        l += r[a.rows * D + a.rows + h] * f;
      }
      if (flag == 3) {
        y[x] = __float2half_rn(o / l);
      } else {
        out[x] = o;
        if (x % D == 0) {
          out[a.rows * D + h] = m;
          out[a.rows * D + a.rows + h] = l;
        }
      }
    }
    if (flag != 3) {                                        // the segment reaches into other CTAs
      const long long n = tiles_of(b);
      const long long from = start_of_sequence(b) * a.units + unit * n;
      // CTA i starts at tile floor(i * all / ctas)
      const int c0 = int(((from + 1) * ctas + all - 1) / all) - 1, c1 = int(((from + n) * ctas + all - 1) / all) - 1;
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        // the count of a segment starts with the first arrival of this call: whatever the word held before
        unsigned long long* word = a.arrived + seg;
        unsigned long long old = *reinterpret_cast<volatile unsigned long long*>(word), was, now;
        do {
          was = old;
          now = (was >> 16) == (a.tag >> 16) ? was + 1 : a.tag + 1;
          if (int(now & 0xFFFFu) == c1 - c0 + 1) now = 0;   // the last: a replay of the same launch starts anew
          old = atomicCAS(word, was, now);
        } while (old != was);
        s_last = now == 0;
      }
      __syncthreads();
      if (s_last) {
        __threadfence();
        for (int x = tid; x < rows * D; x += kDecodeThreads) {
          const int h = x / D;
          float m = -INFINITY, l = 0.0f, o = 0.0f;
#pragma unroll 4
          for (int i = c0; i <= c1; ++i) {
            const float* r = a.records + (int64_t(i) * 2 + (i == c0 ? 1 : 0)) * record;
            const float rm = __ldcg(r + a.rows * D + h), rl = __ldcg(r + a.rows * D + a.rows + h), ro = __ldcg(r + x);
            const float to = fmaxf(m, rm);
            const float ref = to == -INFINITY ? 0.0f : to;
            const float f0 = exp2_fast(m - ref), f1 = exp2_fast(rm - ref);
            o = o * f0 + ro * f1;
            l = l * f0 + rl * f1;
            m = to;
          }
          y[x] = __float2half_rn(o / l);
        }
      }
      __syncthreads();
    }
    i0 = i1;
  }
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
  const int smem = kWarps * (S::kWarpBytes + a.rows * (D + 2) * 4);
  const void* kern = reinterpret_cast<const void*>(&attn_decode_kernel<D, kBits, NT>);
  if (!allow_dynamic_smem(kern, kWarps * (S::kWarpBytes + S::kRecord * 4))) return SMOOTHROT_CUDA_ERROR;
  attn_decode_kernel<D, kBits, NT><<<unsigned(device_sm_count() * S::kCtas), kDecodeThreads, smem, st>>>(a, c);
  count_launch();
  return launch_status();
}

}  // namespace paged
}  // namespace smoothrot

extern "C" {

int smoothrot_decode_status_word(int* out, int clear) {
  return smoothrot::paged::read_status_word(smoothrot::paged::g_decode_status, out, clear);
}

size_t smoothrot_attn_decode_workspace_bytes(int64_t B, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim) {
  using namespace smoothrot::paged;
  if (B <= 0 || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads != 0 || head_dim <= 0) return 0;
  DecodeArgs a;
  decode_plan(n_heads, n_kv_heads, &a);
  const int64_t words = (B * a.units * 8 + 15) / 16 * 16;
  return size_t(words + decode_grid() * 2 * a.rows * (head_dim + 2) * 4);
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
  if (max_pages * page_size > INT32_MAX || B * max_pages * page_size > (int64_t(1) << 34)) return SMOOTHROT_INVALID_ARG;
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
  a.records = reinterpret_cast<float*>(static_cast<char*>(workspace) + (B * a.units * 8 + 15) / 16 * 16);
  static std::atomic<unsigned long long> calls{0x5A17C0DEull};
  a.tag = (calls.fetch_add(1, std::memory_order_relaxed) * 0x9E3779B97F4A7C15ull | (1ull << 63)) & ~0xFFFFull;
  Cache c = make_cache(n_kv_heads, head_dim, bits, pages, page_size, k_cache, v_cache, k_params, v_params);
  if (pages == 0) {           // no page is valid; the copies of nothing still name an address
    c.k = c.v = workspace;
    c.k_params = c.v_params = static_cast<float2*>(workspace);
  }
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
