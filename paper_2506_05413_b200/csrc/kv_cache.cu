// The paged key-value cache of libsmoothrot: tokens appended with the position rotation on the way, and
// rows read back (layout: paged.cuh; codec of the 4-bit form: kv_quant.cu, Eq. 1's asymmetric form).
//
// Both kernels stream: half a warp owns 128 consecutive values of a token's row (one head of 128 or
// two of 64), a lane 8 of them, i.e. one 16-byte load or store of fp16.
//
// Measured (device time; floor at 6552 GB/s in brackets).  Append: 8192 tokens of 32 + 32 + 32 fp16 heads 83 us (61), 2048 of
// 32 + 8 + 8 into 4 bits 18.0 us (6.7), 61 tokens 3.5 us, one 3.1 us.  It is bound by its instructions: 5200 a token of 48 heads
// across its warps, two heads an instruction, at two thirds of the issue slots (profiled at 2048 tokens).
// Gather: 8192 tokens of 32 fp16 heads 43.5 us (41), at the memory's rate; 16384 of 8 heads in 4 bits 19.2 us (13.1).
#include "paged.cuh"
#include "rowquant.cuh"

namespace smoothrot {
namespace paged {

__device__ int g_cache_status = 0;

constexpr int kThreads = 256;
constexpr int kHalfWarps = kThreads / 16;

__device__ __forceinline__ void unpack8(const uint4& raw, float (&v)[8]) {
  const __half2* h = reinterpret_cast<const __half2*>(&raw);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(h[i]);
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  uint4 raw;
  __half2* h = reinterpret_cast<__half2*>(&raw);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
  return raw;
}

// Products of two pairs, each rounded to fp32.  Not mul2: the compiler may make one fma of a packed product and the packed
// sum that takes it, and the rotation and the codes are defined with the product rounded by itself (a
// code at a rounding boundary moves with it).
__device__ __forceinline__ f32x2 rounded_product(f32x2 a, f32x2 b) {
  float a0, a1, b0, b1;
  unpack2(a, a0, a1);
  unpack2(b, b0, b1);
  return pack2(__fmul_rn(a0, b0), __fmul_rn(a1, b1));
}

struct AppendArgs {
  const __half *q, *k, *v;
  int64_t ldq, ldk, ldv;
  __half *q_out, *k_out;
  int64_t ldqo, ldko;
  const int32_t* positions;
  const float* rotary;       // [rotary_rows][D]: D / 2 cosines, then D / 2 sines
  int64_t rotary_rows;
  const int64_t* slots;
  int64_t tokens;
  int q_units, kv_units;     // units of 128 values in a token's queries and in its keys
  int q_values, kv_values;   // values in them (with an odd number of heads of 64 the last unit is half full)
  int walsh, interleaved;
  float clip;
};

constexpr int kBatch = 2;    // pairs of units whose loads a warp has on their way at once

// A warp takes pairs of neighbouring units of one kind (queries, keys or values), a half-warp per unit, so that which
// kind it is does not differ within a warp.  kWarpsPerToken warps share a token's pairs; blockIdx.y splits them further
// where there are few tokens, so that a call for a single token costs one load, one rotation and one
// store in sequence.  A lane keeps its cosines and sines for all units of a token: every unit starts at a
// head's first value, so the lane's place in its head is the same in each.
template <int D, int kBits, int kWarpsPerToken>
__global__ void __launch_bounds__(kThreads, 4)
kv_append_kernel(AppendArgs a, Cache c) {
  constexpr int kTokens = kThreads / 32 / kWarpsPerToken;
  const int lane = threadIdx.x & 31, sub = lane & 15, side = lane >> 4;
  const int warp = (threadIdx.x >> 5) % kWarpsPerToken;
  const int place = (sub * 8) % D;                 // of the lane's first value in its head
  const int q_pairs = (a.q_units + 1) / 2, kv_pairs = (a.kv_units + 1) / 2, pairs = q_pairs + 2 * kv_pairs;
  const int step = gridDim.y * kWarpsPerToken;
  for (int64_t t = int64_t(blockIdx.x) * kTokens + (threadIdx.x >> 5) / kWarpsPerToken; t < a.tokens;
       t += int64_t(gridDim.x) * kTokens) {
    const __half* const q = a.q + t * a.ldq;
    const __half* const k = a.k + t * a.ldk;
    const __half* const v = a.v + t * a.ldv;
    uint4 raws[kBatch];
    auto load = [&](int p0) {
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int p = p0 + b * step;
        const __half* src = p < q_pairs ? q : (p < q_pairs + kv_pairs ? k : v);
        const int first = p < q_pairs ? 0 : (p < q_pairs + kv_pairs ? q_pairs : q_pairs + kv_pairs);
        const int at = (2 * (p - first) + side) * kGroup + sub * 8;
        raws[b] = make_uint4(0, 0, 0, 0);
        if (p < pairs && at < (p < q_pairs ? a.q_values : a.kv_values)) raws[b] = __ldg(reinterpret_cast<const uint4*>(src + at));
      }
    };
    int p0 = blockIdx.y * kWarpsPerToken + warp;
    load(p0);                                      // needs neither the position nor the slot
    const int position = __ldg(a.positions + t);
    const int64_t slot = __ldg(a.slots + t);
    const bool sound = position >= 0 && position < a.rotary_rows && slot < c.pages * c.page_size;
    if (!sound) {                                  // nothing of this token is written
      if (lane == 0) atomicCAS(&g_cache_status, 0, int(kAppendRange));
      continue;
    }
    const bool keep = slot >= 0;                   // a negative slot: rotated, but not cached
    const bool clip_far = a.clip >= 0.5f;          // values reach at most 1 / clip times as far as the clipped range
    // where the token's row of head 0 and its pair of group 0 lie; a page is below 2^31 bytes
    constexpr uint32_t kRow = kBits == 16 ? 2 * D : D / 2;
    const int64_t page = slot >> c.page_shift;
    const int offset = int(slot & (c.page_size - 1));
    const int64_t row0 = head_row(c, page, 0, offset) * kRow + (kBits == 16 ? 2 * place : place / 2), pair0 = param_row(c, page, 0, offset);
    // The rotation of the lane's value x with its partner o: x cos + o (-sin) for the first of a pair, x cos + o sin for the
    // second, each product rounded to fp32.  Packed in twos.
    f32x2 cs[4], sn[4];
    {
      const float* row = a.rotary + int64_t(position) * D;
      if (a.interleaved) {                         // pairs (2 i, 2 i + 1): four angles
        const float4 x = __ldg(reinterpret_cast<const float4*>(row + place / 2));
        const float4 y = __ldg(reinterpret_cast<const float4*>(row + D / 2 + place / 2));
        cs[0] = pack2(x.x, x.x); cs[1] = pack2(x.y, x.y); cs[2] = pack2(x.z, x.z); cs[3] = pack2(x.w, x.w);
        sn[0] = pack2(-y.x, y.x); sn[1] = pack2(-y.y, y.y); sn[2] = pack2(-y.z, y.z); sn[3] = pack2(-y.w, y.w);
      } else {                                     // pairs (i, i + D / 2): eight angles
        const float* at = row + place % (D / 2);
        const float sign = place < D / 2 ? -1.0f : 1.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float4 x = __ldg(reinterpret_cast<const float4*>(at) + i);
          const float4 y = __ldg(reinterpret_cast<const float4*>(at + D / 2) + i);
          cs[2 * i] = pack2(x.x, x.y); cs[2 * i + 1] = pack2(x.z, x.w);
          sn[2 * i] = pack2(sign * y.x, sign * y.y); sn[2 * i + 1] = pack2(sign * y.z, sign * y.w);
        }
      }
    }
    while (p0 < pairs) {
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int p = p0 + b * step;
        if (p >= pairs) break;
        const int kind = p < q_pairs ? 0 : (p < q_pairs + kv_pairs ? 1 : 2);
        const int index = 2 * (p - (kind == 0 ? 0 : (kind == 1 ? q_pairs : q_pairs + kv_pairs))) + side;
        const int at = index * kGroup + sub * 8;
        const bool live = at < (kind == 0 ? a.q_values : a.kv_values);
        uint4 out = raws[b];                       // a value: as it came
        float x[8];
        if (kind != 2) {
          f32x2 y[4], o[4];
          const uint32_t mine[4] = {raws[b].x, raws[b].y, raws[b].z, raws[b].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t other = a.interleaved ? __byte_perm(mine[i], 0, 0x1032) : __shfl_xor_sync(0xffffffffu, mine[i], D / 16);
            y[i] = half2_to_f32x2(mine[i]);
            o[i] = half2_to_f32x2(other);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = add2(rounded_product(y[i], cs[i]), rounded_product(o[i], sn[i]));
          if (a.walsh) {                           // y H_D / sqrt(D), butterflies of stride 1, 2, 4, then between lanes
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float lo, hi;
              unpack2(y[i], lo, hi);
              y[i] = pack2(__fadd_rn(lo, hi), __fsub_rn(lo, hi));
            }
#pragma unroll
            for (int h = 1; h < 4; h <<= 1) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                if ((i & h) == 0) {
                  const f32x2 lo = y[i], hi = y[i + h];
                  y[i] = add2(lo, hi);
                  y[i + h] = sub2(lo, hi);
                }
              }
            }
#pragma unroll
            for (int h = 1; h < D / 8; h <<= 1) {
              // o + y or o - y: the upper lane's own value is taken with the other sign
              const float sign = (sub & h) != 0 ? -1.0f : 1.0f;
              const f32x2 sign2 = pack2(sign, sign);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                float lo, hi;
                unpack2(y[i], lo, hi);
                const f32x2 other = pack2(__shfl_xor_sync(0xffffffffu, lo, h), __shfl_xor_sync(0xffffffffu, hi, h));
                y[i] = fma2(y[i], sign2, other);   // the product with 1 or -1 is exact: one rounding, the sum's
              }
            }
            const float norm = D == 128 ? 0.08838834764831845f : 0.125f;   // 1 / sqrt(D)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = mul2(y[i], pack2(norm, norm));
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) unpack2(y[i], x[2 * i], x[2 * i + 1]);
          out = pack8(x);
        } else if (kBits == 4) {
          unpack8(raws[b], x);
        }
        if (kind == 0) {
          if (live) *reinterpret_cast<uint4*>(a.q_out + t * a.ldqo + at) = out;
          continue;
        }
        if (kind == 1 && a.k_out != nullptr && live) *reinterpret_cast<uint4*>(a.k_out + t * a.ldko + at) = out;
        if (kBits == 16) {
          if (live && keep) {
            char* dst = static_cast<char*>(kind == 1 ? c.k : c.v) + row0;
            *reinterpret_cast<uint4*>(dst + (uint32_t(at / D) << c.page_shift) * kRow) = out;
          }
        } else {
          // Eq. 1's asymmetric form on the unit's 128 values, as kv_quant_kernel takes every decision
          float hi = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
          float lo = fminf(fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), fminf(fminf(x[4], x[5]), fminf(x[6], x[7])));
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) {
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
          }
          hi = __fmul_rn(a.clip, hi);
          lo = __fmul_rn(a.clip, lo);
          const float step_size = hi == lo ? 1.0f : __fdiv_rn(__fsub_rn(hi, lo), 15.0f);
          const float zero = -rintf(__fdiv_rn(lo, step_size));
          const float inv = __frcp_rn(step_size);
          uint32_t packed = 0;
          // x / step + zero to the nearest whole number, clamped.  Adding 1.5 * 2^23 rounds to the nearest whole number, ties to
          // even, for magnitudes below 2^22, and the zero point is then added exactly; a group further from
          // zero, in its own steps, takes the long way, which also keeps NaN apart.
          const bool near = fabsf(zero) < 1048576.0f && clip_far;
          if (__all_sync(0xffffffffu, near)) {
            const f32x2 inv2 = pack2(inv, inv), magic2 = pack2(12582912.0f, 12582912.0f), zero2 = pack2(zero, zero);
            uint32_t weight = 1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float u0, u1;
              unpack2(add2(add2(rounded_product(pack2(x[2 * i], x[2 * i + 1]), inv2), magic2), zero2), u0, u1);
              u0 = fminf(fmaxf(u0, 12582912.0f), 12582927.0f);
              u1 = fminf(fmaxf(u1, 12582912.0f), 12582927.0f);
              packed += (__float_as_uint(u0) - 0x4B400000u) * weight;
              packed += (__float_as_uint(u1) - 0x4B400000u) * (weight << 4);
              weight <<= 8;
            }
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float code = fminf(fmaxf(__fadd_rn(rintf(__fmul_rn(x[i], inv)), zero), 0.0f), 15.0f);
              packed |= uint32_t(code) << (4 * i);
            }
          }
          if (live && keep) {
            char* dst = static_cast<char*>(kind == 1 ? c.k : c.v) + row0;
            *reinterpret_cast<uint32_t*>(dst + (uint32_t(at / D) << c.page_shift) * kRow) = packed;
            if (sub == 0) ((kind == 1 ? c.k_params : c.v_params) + pair0)[uint32_t(index) << c.page_shift] = make_float2(step_size, zero);
          }
        }
      }
      p0 += kBatch * step;
      if (p0 < pairs) load(p0);
    }
  }
}

struct GatherArgs {
  const int64_t* slots;
  int64_t tokens;
  int units;
  int values;
  __half *k_out, *v_out;
  int64_t ldk, ldv;
};

// One half-warp per (token, unit), keys and values together; kItems of them at a time, their slots first, then all their
// loads, so that a lane has 2 * kItems loads on their way.
template <int D, int kBits, int kItems>
__global__ void __launch_bounds__(kThreads)
kv_gather_kernel(GatherArgs a, Cache c) {
  const int sub = threadIdx.x & 15;
  const uint32_t total = uint32_t(a.tokens) * uint32_t(a.units);
  const uint32_t first = blockIdx.x * (kHalfWarps * kItems) + (threadIdx.x >> 4);
  int64_t slot[kItems];
  int at[kItems];
  uint32_t token[kItems];
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const uint32_t i = first + k * kHalfWarps;
    token[k] = i / uint32_t(a.units);
    at[k] = int(i - token[k] * uint32_t(a.units)) * kGroup + sub * 8;
    if (i >= total) at[k] = a.values;                // nothing to do
    slot[k] = at[k] < a.values ? __ldg(a.slots + token[k]) : -1;
    if (slot[k] >= c.pages * c.page_size) {
      if (sub == 0) atomicCAS(&g_cache_status, 0, int(kGatherRange));
      slot[k] = -1;
    }
  }
  if (kBits == 16) {
    uint4 ko[kItems], vo[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      ko[k] = vo[k] = make_uint4(0, 0, 0, 0);        // a negative slot: zeros
      if (slot[k] < 0) continue;
      const int64_t row = head_row(c, slot[k] >> c.page_shift, at[k] / D, int(slot[k] & (c.page_size - 1))) * D + at[k] % D;
      ko[k] = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __half*>(c.k) + row));
      vo[k] = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __half*>(c.v) + row));
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      if (at[k] >= a.values) continue;
      *reinterpret_cast<uint4*>(a.k_out + int64_t(token[k]) * a.ldk + at[k]) = ko[k];
      *reinterpret_cast<uint4*>(a.v_out + int64_t(token[k]) * a.ldv + at[k]) = vo[k];
    }
  } else {
    uint32_t kc[kItems], vc[kItems];
    float2 kp[kItems], vp[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      kc[k] = vc[k] = 0;
      kp[k] = vp[k] = make_float2(0.0f, 0.0f);
      if (slot[k] < 0) continue;
      const int64_t page = slot[k] >> c.page_shift;
      const int offset = int(slot[k] & (c.page_size - 1));
      const int64_t row = head_row(c, page, at[k] / D, offset) * (D / 2) + at[k] % D / 2;
      const int64_t group = param_row(c, page, at[k] / kGroup, offset);
      kc[k] = __ldg(reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(c.k) + row));
      vc[k] = __ldg(reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(c.v) + row));
      kp[k] = __ldg(c.k_params + group);
      vp[k] = __ldg(c.v_params + group);
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      if (at[k] >= a.values) continue;
      float x[8], y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = __fmul_rn(__fsub_rn(float((kc[k] >> (4 * j)) & 15u), kp[k].y), kp[k].x);
        y[j] = __fmul_rn(__fsub_rn(float((vc[k] >> (4 * j)) & 15u), vp[k].y), vp[k].x);
      }
      *reinterpret_cast<uint4*>(a.k_out + int64_t(token[k]) * a.ldk + at[k]) = pack8(x);
      *reinterpret_cast<uint4*>(a.v_out + int64_t(token[k]) * a.ldv + at[k]) = pack8(y);
    }
  }
}

// Warps a token and pairs a batch, swept together (2048 tokens in 4 bits / 8192 of 32 heads in fp16, us, 4 blocks an SM): 2 and
// 2: 17.2 / 81.8, 1 and 2: 21.8 / 80.8, 2 and 3: 18.0 / 79.2; with 8 warps a token and no bound on registers 25 / 113.
constexpr int kManyWarps = 2;
template <int D, int kBits>
static void launch_append(const AppendArgs& a, const Cache& c, cudaStream_t st) {
  const int64_t sms = device_sm_count();
  const int pairs = (a.q_units + 1) / 2 + (a.kv_units + 1) / 2 * 2;
  if (a.tokens <= sms * 4) {
    // Few tokens: a warp per pair of units.  With Walsh, this form / the other, us: 32 + 8 heads of 128 in 4 bits, 1 token 2.6 / 8.0,
    // 148 3.8 / 9.4, 592 9.0 / 9.6, 740 11.0 / 12.1, 888 12.6 / 12.0, 1184 15.9 / 12.1; 32 + 32 heads in fp16, 1 token 2.6 / 12.0,
    // 592 13.7 / 13.6, 888 19.4 / 16.7; 12 + 4 heads of 64 in 4 bits, 592 3.7 / 3.8, 740 5.2 / 4.2.
    const unsigned split = unsigned((pairs + 7) / 8);
    kv_append_kernel<D, kBits, 8><<<dim3(unsigned(a.tokens), split > 65535u ? 65535u : split), kThreads, 0, st>>>(a, c);
  } else {
    constexpr int kTokens = kThreads / 32 / kManyWarps;
    const int64_t want = (a.tokens + kTokens - 1) / kTokens, most = sms * 128;
    kv_append_kernel<D, kBits, kManyWarps><<<unsigned(want < most ? want : most), kThreads, 0, st>>>(a, c);
  }
}

// Two items a half-warp, or one where all of them run at once (777 tokens of 4 heads of 64: 2.8 us with one, 2.8 with
// two, 4.1 with four; 16384 tokens of 8 heads in 4 bits: 21.9, 19.8, 20.5).
template <int D, int kBits>
static void launch_gather(const GatherArgs& a, const Cache& c, cudaStream_t st) {
  const int64_t items = a.tokens * a.units;
  if (items <= int64_t(device_sm_count()) * 8 * kHalfWarps)
    kv_gather_kernel<D, kBits, 1><<<unsigned((items + kHalfWarps - 1) / kHalfWarps), kThreads, 0, st>>>(a, c);
  else
    kv_gather_kernel<D, kBits, 2><<<unsigned((items + 2 * kHalfWarps - 1) / (2 * kHalfWarps)), kThreads, 0, st>>>(a, c);
}

}  // namespace paged
}  // namespace smoothrot

extern "C" {

int smoothrot_cache_status_word(int* out, int clear) {
  return smoothrot::paged::read_status_word(smoothrot::paged::g_cache_status, out, clear);
}

int smoothrot_kv_append(const void* Q_f16, int64_t ldq, const void* K_f16, int64_t ldk, const void* V_f16, int64_t ldv,
                        int64_t T, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim, const int32_t* positions,
                        const float* rotary, int64_t rotary_rows, int interleaved, int walsh, void* Q_out_f16,
                        int64_t ldqo, void* K_out_f16, int64_t ldko, const int64_t* slots, int bits, int64_t pages,
                        int64_t page_size, void* k_cache, void* v_cache, float* k_params, float* v_params, float clip,
                        void* stream) {
  using namespace smoothrot;
  using namespace smoothrot::paged;
  if (T < 0 || n_heads < 0 || n_heads > 65535 || rotary_rows < 0) return SMOOTHROT_INVALID_ARG;
  const int sizes = check_sizes(n_kv_heads, head_dim, bits, pages, page_size);
  if (sizes != SMOOTHROT_OK) return sizes;
  if (!(clip > 0.0f) || clip > 1.0f) return SMOOTHROT_INVALID_ARG;
  if ((interleaved & ~1) != 0 || (walsh & ~1) != 0) return SMOOTHROT_INVALID_ARG;
  if (T == 0) return SMOOTHROT_OK;
  const int64_t cq = n_heads * head_dim, ckv = n_kv_heads * head_dim;
  if (K_f16 == nullptr || V_f16 == nullptr || positions == nullptr || rotary == nullptr || slots == nullptr)
    return SMOOTHROT_INVALID_ARG;
  if (ldk < ckv || ldv < ckv || (K_out_f16 != nullptr && ldko < ckv)) return SMOOTHROT_INVALID_ARG;
  if (n_heads > 0 && (Q_f16 == nullptr || Q_out_f16 == nullptr || ldq < cq || ldqo < cq)) return SMOOTHROT_INVALID_ARG;
  const int pointers = check_pointers(bits, k_cache, v_cache, k_params, v_params);
  if (pointers != SMOOTHROT_OK) return pointers;
  if (!aligned16(K_f16) || !aligned16(V_f16) || !aligned16(rotary) || ldk % 8 != 0 || ldv % 8 != 0) return SMOOTHROT_BAD_ALIGNMENT;
  if (K_out_f16 != nullptr && (!aligned16(K_out_f16) || ldko % 8 != 0)) return SMOOTHROT_BAD_ALIGNMENT;
  if (n_heads > 0 && (!aligned16(Q_f16) || !aligned16(Q_out_f16) || ldq % 8 != 0 || ldqo % 8 != 0)) return SMOOTHROT_BAD_ALIGNMENT;
  AppendArgs a;
  a.q = static_cast<const __half*>(Q_f16); a.k = static_cast<const __half*>(K_f16); a.v = static_cast<const __half*>(V_f16);
  a.ldq = ldq; a.ldk = ldk; a.ldv = ldv;
  a.q_out = static_cast<__half*>(Q_out_f16); a.k_out = static_cast<__half*>(K_out_f16);
  a.ldqo = ldqo; a.ldko = ldko;
  a.positions = positions; a.rotary = rotary; a.rotary_rows = rotary_rows; a.slots = slots;
  a.tokens = T;
  a.q_values = int(cq); a.kv_values = int(ckv);
  a.q_units = int((cq + kGroup - 1) / kGroup); a.kv_units = int((ckv + kGroup - 1) / kGroup);
  a.walsh = walsh; a.interleaved = interleaved; a.clip = clip;
  const Cache c = make_cache(n_kv_heads, head_dim, bits, pages, page_size, k_cache, v_cache, k_params, v_params);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (head_dim == 128) {
    if (bits == 16) launch_append<128, 16>(a, c, st);
    else launch_append<128, 4>(a, c, st);
  } else {
    if (bits == 16) launch_append<64, 16>(a, c, st);
    else launch_append<64, 4>(a, c, st);
  }
  count_launch();
  return launch_status();
}

int smoothrot_kv_gather(const int64_t* slots, int64_t T, int64_t n_kv_heads, int64_t head_dim, int bits, int64_t pages,
                        int64_t page_size, const void* k_cache, const void* v_cache, const float* k_params,
                        const float* v_params, void* K_out_f16, int64_t ldk, void* V_out_f16, int64_t ldv, void* stream) {
  using namespace smoothrot;
  using namespace smoothrot::paged;
  if (T < 0) return SMOOTHROT_INVALID_ARG;
  const int sizes = check_sizes(n_kv_heads, head_dim, bits, pages, page_size);
  if (sizes != SMOOTHROT_OK) return sizes;
  if (T == 0) return SMOOTHROT_OK;
  const int64_t ckv = n_kv_heads * head_dim;
  const int64_t units = (ckv + kGroup - 1) / kGroup;
  if (T > INT32_MAX / units) return SMOOTHROT_INVALID_ARG;
  if (slots == nullptr || K_out_f16 == nullptr || V_out_f16 == nullptr || ldk < ckv || ldv < ckv) return SMOOTHROT_INVALID_ARG;
  const int pointers = check_pointers(bits, k_cache, v_cache, k_params, v_params);
  if (pointers != SMOOTHROT_OK) return pointers;
  if (!aligned16(K_out_f16) || !aligned16(V_out_f16) || ldk % 8 != 0 || ldv % 8 != 0) return SMOOTHROT_BAD_ALIGNMENT;
  GatherArgs a;
  a.slots = slots; a.tokens = T; a.units = int(units); a.values = int(ckv);
  a.k_out = static_cast<__half*>(K_out_f16); a.v_out = static_cast<__half*>(V_out_f16);
  a.ldk = ldk; a.ldv = ldv;
  const Cache c = make_cache(n_kv_heads, head_dim, bits, pages, page_size, k_cache, v_cache, k_params, v_params);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (head_dim == 128) {
    if (bits == 16) launch_gather<128, 16>(a, c, st);
    else launch_gather<128, 4>(a, c, st);
  } else {
    if (bits == 16) launch_gather<64, 16>(a, c, st);
    else launch_gather<64, 4>(a, c, st);
  }
  count_launch();
  return launch_status();
}

}  // extern "C"
