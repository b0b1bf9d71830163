// The paged key-value cache of libsmoothrot: tokens appended with the position rotation on the way, and
// rows read back (layout: paged.cuh; codec of the 4-bit form: kv_quant.cu, Eq. 1's asymmetric form).
//
// Both kernels stream: half a warp owns 128 consecutive values of a token's row (one head of 128 or
// two of 64), a lane 8 of them, i.e. one 16-byte load or store of fp16.
#include "paged.cuh"

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

// One half-warp per unit; blockIdx.y splits a token's units where there are few tokens, so that a call for a
// single token costs one load, one rotation and one store in sequence.  With many tokens a lane keeps its
// cosines and sines for all units of a token (every unit starts at a head's first value, so the
// lane's place in its head is the same in each).
template <int D, int kBits>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(AppendArgs a, Cache c) {
  const int sub = threadIdx.x & 15;
  const int half_warp = threadIdx.x >> 4;
  const int place = (sub * 8) % D;                 // of the lane's first value in its head
  const int units = a.q_units + 2 * a.kv_units;
  for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
    const int position = a.positions[t];
    const int64_t slot = a.slots[t];
    const bool sound = position >= 0 && position < a.rotary_rows && slot < c.pages * c.page_size;
    if (!sound) {                                  // nothing of this token is written
      if (threadIdx.x == 0) atomicCAS(&g_cache_status, 0, int(kAppendRange));
      continue;
    }
    const bool keep = slot >= 0;                   // a negative slot: rotated, but not cached
    const int64_t page = slot >> c.page_shift;
    const int offset = int(slot & (c.page_size - 1));
    float cs[8], sn[8];
    {
      const float* row = a.rotary + int64_t(position) * D;
      if (a.interleaved) {                         // pairs (2 i, 2 i + 1): four angles
        const float4 x = __ldg(reinterpret_cast<const float4*>(row + place / 2));
        const float4 y = __ldg(reinterpret_cast<const float4*>(row + D / 2 + place / 2));
        cs[0] = cs[1] = x.x; cs[2] = cs[3] = x.y; cs[4] = cs[5] = x.z; cs[6] = cs[7] = x.w;
        sn[0] = sn[1] = y.x; sn[2] = sn[3] = y.y; sn[4] = sn[5] = y.z; sn[6] = sn[7] = y.w;
      } else {                                     // pairs (i, i + D / 2): eight angles
        const float* at = row + place % (D / 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float4 x = __ldg(reinterpret_cast<const float4*>(at) + i);
          const float4 y = __ldg(reinterpret_cast<const float4*>(at + D / 2) + i);
          cs[4 * i] = x.x; cs[4 * i + 1] = x.y; cs[4 * i + 2] = x.z; cs[4 * i + 3] = x.w;
          sn[4 * i] = y.x; sn[4 * i + 1] = y.y; sn[4 * i + 2] = y.z; sn[4 * i + 3] = y.w;
        }
      }
    }
    // whole warps stay together (shuffles): the loop runs over pairs of units
    for (int u0 = blockIdx.y * kHalfWarps + (half_warp & ~1); u0 < units; u0 += gridDim.y * kHalfWarps) {
      const int u = u0 + (half_warp & 1);
      const int part = u < a.q_units ? 0 : (u < a.q_units + a.kv_units ? 1 : 2);      // query, key or value
      const int w = u - (part == 0 ? 0 : (part == 1 ? a.q_units : a.q_units + a.kv_units));
      const int at = w * kGroup + sub * 8;
      const bool live = u < units && at < (part == 0 ? a.q_values : a.kv_values);
      const __half* src = part == 0 ? a.q + t * a.ldq : (part == 1 ? a.k + t * a.ldk : a.v + t * a.ldv);
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (live) raw = __ldg(reinterpret_cast<const uint4*>(src + at));
      float x[8];
      unpack8(raw, x);
      // The rotation of pair (a, b): a c - b s and b c + a s, each product rounded to fp32.  All lanes take
      // part in the shuffles; a value unit keeps what it had.
      float y[8];
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          y[i] = __fsub_rn(__fmul_rn(x[i], cs[i]), __fmul_rn(x[i + 1], sn[i]));
          y[i + 1] = __fadd_rn(__fmul_rn(x[i + 1], cs[i]), __fmul_rn(x[i], sn[i]));
        }
      } else {
        uint4 other;
        other.x = __shfl_xor_sync(0xffffffffu, raw.x, D / 16);
        other.y = __shfl_xor_sync(0xffffffffu, raw.y, D / 16);
        other.z = __shfl_xor_sync(0xffffffffu, raw.z, D / 16);
        other.w = __shfl_xor_sync(0xffffffffu, raw.w, D / 16);
        float o[8];
        unpack8(other, o);
        const bool first = place < D / 2;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float turn = __fmul_rn(o[i], sn[i]);
          y[i] = first ? __fsub_rn(__fmul_rn(x[i], cs[i]), turn) : __fadd_rn(__fmul_rn(x[i], cs[i]), turn);
        }
      }
      if (a.walsh) {                               // y H_D / sqrt(D), butterflies of stride 1, 2, 4, then between lanes
#pragma unroll
        for (int h = 1; h < 8; h <<= 1) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if ((i & h) == 0) {
              const float lo = y[i], hi = y[i + h];
              y[i] = __fadd_rn(lo, hi);
              y[i + h] = __fsub_rn(lo, hi);
            }
          }
        }
#pragma unroll
        for (int h = 1; h < D / 8; h <<= 1) {
          const bool up = (sub & h) != 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float o = __shfl_xor_sync(0xffffffffu, y[i], h);
            y[i] = up ? __fsub_rn(o, y[i]) : __fadd_rn(y[i], o);
          }
        }
        const float norm = D == 128 ? 0.08838834764831845f : 0.125f;   // 1 / sqrt(D)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __fmul_rn(y[i], norm);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = part == 2 ? x[i] : y[i];
      if (part == 0) {
        if (live) *reinterpret_cast<uint4*>(a.q_out + t * a.ldqo + at) = pack8(x);
      } else if (part == 1 && a.k_out != nullptr) {
        if (live) *reinterpret_cast<uint4*>(a.k_out + t * a.ldko + at) = pack8(x);
      }
      if (kBits == 16) {
        if (part != 0 && live && keep) {
          __half* dst = reinterpret_cast<__half*>(part == 1 ? c.k : c.v) + head_row(c, page, at / D, offset) * D + place;
          *reinterpret_cast<uint4*>(dst) = pack8(x);
        }
      } else {
        // Eq. 1's asymmetric form on the unit's 128 values, as kv_quant_kernel takes every decision
        float hi = x[0], lo = x[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) {
          hi = fmaxf(hi, x[i]);
          lo = fminf(lo, x[i]);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
          hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
          lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        }
        hi = __fmul_rn(a.clip, hi);
        lo = __fmul_rn(a.clip, lo);
        const float step = hi == lo ? 1.0f : __fdiv_rn(__fsub_rn(hi, lo), 15.0f);
        const float zero = -rintf(__fdiv_rn(lo, step));
        const float inv = __frcp_rn(step);
        uint32_t packed = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float code = fminf(fmaxf(__fadd_rn(rintf(__fmul_rn(x[i], inv)), zero), 0.0f), 15.0f);
          packed |= uint32_t(code) << (4 * i);
        }
        if (part != 0 && live && keep) {
          uint8_t* dst = reinterpret_cast<uint8_t*>(part == 1 ? c.k : c.v) + head_row(c, page, at / D, offset) * (D / 2);
          *reinterpret_cast<uint32_t*>(dst + place / 2) = packed;
          if (sub == 0) (part == 1 ? c.k_params : c.v_params)[param_row(c, page, w, offset)] = make_float2(step, zero);
        }
      }
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

// One half-warp per (token, unit), keys and values together; both loads are on their way before either is used.
template <int D, int kBits>
__global__ void __launch_bounds__(kThreads)
kv_gather_kernel(GatherArgs a, Cache c) {
  const int sub = threadIdx.x & 15;
  const uint32_t total = uint32_t(a.tokens) * uint32_t(a.units);
  const uint32_t stride = gridDim.x * kHalfWarps;
  for (uint32_t i = blockIdx.x * kHalfWarps + (threadIdx.x >> 4); i < total; i += stride) {
    const uint32_t t = i / uint32_t(a.units);
    const int w = int(i - t * uint32_t(a.units));
    const int at = w * kGroup + sub * 8;
    if (at >= a.values) continue;
    const int64_t slot = a.slots[t];
    uint4 ko = make_uint4(0, 0, 0, 0), vo = ko;      // a negative slot: zeros
    if (slot >= c.pages * c.page_size) {
      if (sub == 0) atomicCAS(&g_cache_status, 0, int(kGatherRange));
    } else if (slot >= 0) {
      const int64_t page = slot >> c.page_shift;
      const int offset = int(slot & (c.page_size - 1));
      const int64_t row = head_row(c, page, at / D, offset);
      if (kBits == 16) {
        ko = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __half*>(c.k) + row * D + at % D));
        vo = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __half*>(c.v) + row * D + at % D));
      } else {
        const uint32_t kc = __ldg(reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(c.k) + row * (D / 2) + at % D / 2));
        const uint32_t vc = __ldg(reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(c.v) + row * (D / 2) + at % D / 2));
        const float2 kp = __ldg(c.k_params + param_row(c, page, w, offset));
        const float2 vp = __ldg(c.v_params + param_row(c, page, w, offset));
        float x[8], y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = __fmul_rn(__fsub_rn(float((kc >> (4 * j)) & 15u), kp.y), kp.x);
          y[j] = __fmul_rn(__fsub_rn(float((vc >> (4 * j)) & 15u), vp.y), vp.x);
        }
        ko = pack8(x);
        vo = pack8(y);
      }
    }
    *reinterpret_cast<uint4*>(a.k_out + int64_t(t) * a.ldk + at) = ko;
    *reinterpret_cast<uint4*>(a.v_out + int64_t(t) * a.ldv + at) = vo;
  }
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
  const int units = a.q_units + 2 * a.kv_units;
  const int64_t resident = int64_t(device_sm_count()) * 8;
  // few tokens: one unit per half-warp, many: one block per token
  const unsigned split = T * 2 <= resident ? unsigned((units + kHalfWarps - 1) / kHalfWarps) : 1u;
  const int64_t blocks = T < resident * 16 ? T : resident * 16;
  const dim3 grid(unsigned(blocks), split > 65535u ? 65535u : split);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (head_dim == 128) {
    if (bits == 16) kv_append_kernel<128, 16><<<grid, kThreads, 0, st>>>(a, c);
    else kv_append_kernel<128, 4><<<grid, kThreads, 0, st>>>(a, c);
  } else {
    if (bits == 16) kv_append_kernel<64, 16><<<grid, kThreads, 0, st>>>(a, c);
    else kv_append_kernel<64, 4><<<grid, kThreads, 0, st>>>(a, c);
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
  const int64_t want = (T * units + kHalfWarps - 1) / kHalfWarps;
  const int64_t cap = int64_t(device_sm_count()) * 8 * 4;
  const unsigned grid = unsigned(want < cap ? want : cap);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (head_dim == 128) {
    if (bits == 16) kv_gather_kernel<128, 16><<<grid, kThreads, 0, st>>>(a, c);
    else kv_gather_kernel<128, 4><<<grid, kThreads, 0, st>>>(a, c);
  } else {
    if (bits == 16) kv_gather_kernel<64, 16><<<grid, kThreads, 0, st>>>(a, c);
    else kv_gather_kernel<64, 4><<<grid, kThreads, 0, st>>>(a, c);
  }
  count_launch();
  return launch_status();
}

}  // extern "C"
