// The residual stream between two blocks: a block's output, normalised and gated, added to the stream, and the norm in
// front of the next block with that block's quantizer behind it.
//
//   z  = y                         or  y * rstd(y) * post_w
//   h' = fp16(residual_scale * h + block_scale * gate * z)
//   x  = fp16(h' * rstd(h') * pre_w)           rstd(r) = 1 / sqrt(mean(r^2) + eps)
//   x, and / or its codes: one step per row as in smoothrot_quant_act_plain, or microscaled as in smoothrot_mx_quant
//
// One pass: a row is read once (4 bytes a value), lives in registers as fp16 through both norms and leaves as h' and x
// or codes.  A CTA takes a row at a time, a thread up to 4 chunks of 8 neighbouring values.  Every product and sum of the
// formulas is rounded by itself and the norms' statistics are good to 2^-45 (SquareSum) and rounded once to
// fp32, so the results do not hang on how a row is shared out, and the codes are those of the quantizer run on x.
#include "mx.cuh"

namespace smoothrot {
namespace mx {
namespace {

constexpr int kMaxThreads = 1024;
constexpr int64_t kMaxWidth = 8 * 4 * kMaxThreads;

struct NormArgs {
  const __half *y, *h;
  int64_t ldy, ldh, ldho, ldxo;
  int rows, K;
  const float *post_w, *gate, *pre_w;
  int post_norm;
  float block_scale, residual_scale;
  double eps, inv_k;
  __half *h_out, *x_out;
  float clip;
  uint8_t *q_out, *scale_out;
  float* step_out;
};

// 1 / sqrt(mean + eps) to fp32: a first value from the fp32 approximation, one Newton step in 64 bits.
__device__ __forceinline__ float rstd_of(double sum, double inv_k, double eps) {
  const double a = sum * inv_k + eps;
  const float f = float(a);
  if (!(f >= 1e-37f) || !(f < 1e37f)) return float(rsqrt(a));      // beyond the approximation's range: infinities, NaN
  const double r = double(rsqrtf(f));
  return float(r * (1.5 - 0.5 * a * r * r));
}

template <typename Tv>
__device__ __forceinline__ Tv shfl_sum(Tv v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum over the CTA; `slot` holds a value per warp and is not used again before every thread has passed another barrier.
__device__ __forceinline__ double block_sum(double v, double* slot) {
  v = shfl_sum(v);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return v;
  if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = slot[0];
  for (int w = 1; w < warps; ++w) s += slot[w];
  return s;
}
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* slot) {
  v = __reduce_max_sync(0xffffffffu, v);
  const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  if (warps == 1) return v;
  if (lane == 0) slot[threadIdx.x >> 5] = v;
  __syncthreads();
  return __reduce_max_sync(0xffffffffu, lane < warps ? slot[lane] : 0u);
}

__device__ __forceinline__ void load8(const float* p, int chunk, float (&w)[8]) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p) + 2 * chunk), b = __ldg(reinterpret_cast<const float4*>(p) + 2 * chunk + 1);
  w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
  w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
}
__device__ __forceinline__ void widen8(const uint4& r, float (&v)[8]) {
  unpack2(half2_to_f32x2(r.x), v[0], v[1]);
  unpack2(half2_to_f32x2(r.y), v[2], v[3]);
  unpack2(half2_to_f32x2(r.z), v[4], v[5]);
  unpack2(half2_to_f32x2(r.w), v[6], v[7]);
}
__device__ __forceinline__ uint4 narrow8(const float (&v)[8]) {
  uint4 o;
  __half2* h = reinterpret_cast<__half2*>(&o);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
  return o;
}
__device__ __forceinline__ void square8(SquareSum& s, const uint4& r) {
  s.add(half2_to_f32x2(r.x));
  s.add(half2_to_f32x2(r.y));
  s.add(half2_to_f32x2(r.z));
  s.add(half2_to_f32x2(r.w));
}

// CODES: 0 none, 4 one step per row, 16 and 32 microscaled groups.
template <int CODES, int CH>
__global__ void __launch_bounds__(kMaxThreads) add_norm_kernel(const NormArgs a) {
  __shared__ double sums[2][2][kMaxThreads / 32];
  __shared__ uint32_t tops[2][kMaxThreads / 32];
  const int t = threadIdx.x, T = blockDim.x, lane = t & 31;
  const int chunks = a.K >> 3;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  uint4 y[CH], h[CH];
  auto fetch = [&](int m) {
    const uint4* ys = reinterpret_cast<const uint4*>(a.y + int64_t(m) * a.ldy);
    const uint4* hs = reinterpret_cast<const uint4*>(a.h + int64_t(m) * a.ldh);
#pragma unroll
    for (int c = 0; c < CH; ++c) y[c] = a.y != nullptr && t + c * T < chunks ? __ldcs(ys + t + c * T) : zero;
#pragma unroll
    for (int c = 0; c < CH; ++c) h[c] = a.h != nullptr && t + c * T < chunks ? __ldcs(hs + t + c * T) : zero;
  };
  int m = blockIdx.x;
  after_the_call_before();
  if (m < a.rows) fetch(m);
  // the sums' slots of one row and the next are two sets in turn
  for (int parity = 0; m < a.rows; m += gridDim.x, parity ^= 1) {
    float rstd = 1.0f;
    if (a.post_norm) {
      SquareSum s;
      s.clear();
#pragma unroll
      for (int c = 0; c < CH; ++c) square8(s, y[c]);
      rstd = rstd_of(block_sum(s.total(), sums[parity][0]), a.inv_k, a.eps);
    }
    uint4 kept[CH];
    SquareSum s;
    s.clear();
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int chunk = t + c * T;
      kept[c] = zero;
      if (chunk < chunks) {
        float z[8], r[8], w[8];
        widen8(h[c], r);
        widen8(y[c], z);
        if (a.post_norm) {
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = __fmul_rn(z[i], rstd);
          if (a.post_w != nullptr) {
            load8(a.post_w, chunk, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = __fmul_rn(z[i], w[i]);
          }
        }
        if (a.gate != nullptr) {
          load8(a.gate, chunk, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = __fmul_rn(z[i], w[i]);
        }
        if (a.y == nullptr) {
#pragma unroll
          for (int i = 0; i < 8; ++i) r[i] = __fmul_rn(r[i], a.residual_scale);
        } else if (a.h == nullptr) {
#pragma unroll
          for (int i = 0; i < 8; ++i) r[i] = __fmul_rn(z[i], a.block_scale);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            r[i] = __fadd_rn(__fmul_rn(r[i], a.residual_scale), __fmul_rn(z[i], a.block_scale));
        }
        kept[c] = narrow8(r);
        if (a.h_out != nullptr) __stcs(reinterpret_cast<uint4*>(a.h_out + int64_t(m) * a.ldho) + chunk, kept[c]);
        square8(s, kept[c]);
      }
    }
    if (m + int(gridDim.x) < a.rows) fetch(m + gridDim.x);      // on its way during the second norm
    if (CODES == 0 && a.x_out == nullptr) continue;
    rstd = rstd_of(block_sum(s.total(), sums[parity][1]), a.inv_k, a.eps);
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int chunk = t + c * T;
      if (chunk < chunks) {
        float x[8], w[8];
        widen8(kept[c], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __fmul_rn(x[i], rstd);
        if (a.pre_w != nullptr) {
          load8(a.pre_w, chunk, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = __fmul_rn(x[i], w[i]);
        }
        kept[c] = narrow8(x);
        if (a.x_out != nullptr) __stcs(reinterpret_cast<uint4*>(a.x_out + int64_t(m) * a.ldxo) + chunk, kept[c]);
        if constexpr (CODES == 4 || CODES == 16) {
          widen8(kept[c], x);
#pragma unroll
          for (int i = 0; i < 8; ++i) top = max(top, abs_bits(x[i]));
        }
      }
    }
    if constexpr (CODES == 0) continue;
    float step = 1.0f, inv = 0.0f;
    if constexpr (CODES == 4) {
      step = step_from_absmax(__uint_as_float(block_max(top, tops[parity])), a.clip);
      inv = __frcp_rn(step);
      if (t == 0) a.step_out[m] = step;
    } else if constexpr (CODES == 16) {
      step = row_step_16(block_max(top, tops[parity]));
      if (t == 0) a.step_out[m] = step;
      if (!(step > 0.0f)) step = 1.0f;
    }
    uint32_t* q_row = reinterpret_cast<uint32_t*>(a.q_out + int64_t(m) * (a.K >> 1));
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int chunk = t + c * T;
      float x[8];
      widen8(kept[c], x);
      uint32_t codes = 0, byte = 0, word = 0;
      if constexpr (CODES == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float r = fmaxf(fminf(rintf(quotient(x[i], step, inv)), 7.0f), -8.0f);
          codes |= (uint32_t(int(r)) & 15u) << (4 * i);
        }
      } else if constexpr (CODES == 32) {
        codes = encode_32(x, &byte);
        word = scale_quad<32>(byte, lane);
      } else if constexpr (CODES == 16) {
        codes = encode_16(x, step, &byte);
        word = scale_quad<16>(byte, lane);
      }
      if (chunk < chunks) {
        __stcs(q_row + chunk, codes);
        if constexpr (CODES >= 16)
          if ((lane & (CODES / 2 - 1)) == 0)
            *reinterpret_cast<uint32_t*>(a.scale_out + scale_word(m, chunk / (CODES / 2), chunks / (CODES / 2))) = word;
      }
    }
  }
}

}  // namespace
}  // namespace mx
}  // namespace smoothrot

extern "C" {

int smoothrot_add_norm(const void* Y_f16, int64_t ldy, const void* H_f16, int64_t ldh, int64_t M, int64_t K, int post_norm,
                       const float* post_w, const float* gate, float block_scale, float residual_scale,
                       const float* pre_w, float eps, void* H_out_f16, int64_t ldho, void* X_out_f16, int64_t ldxo,
                       int codes, float clip, uint8_t* q_out, uint8_t* scale_out, float* step_out, void* stream) {
  using namespace smoothrot;
  using namespace smoothrot::mx;
  if (M < 0 || K <= 0 || (post_norm != 0 && post_norm != 1)) return SMOOTHROT_INVALID_ARG;
  if (codes != 0 && codes != 4 && codes != 16 && codes != 32) return SMOOTHROT_INVALID_ARG;
  if (!(eps > 0.0f) || !isfinite(eps) || !isfinite(block_scale) || !isfinite(residual_scale)) return SMOOTHROT_INVALID_ARG;
  if (codes == 4 && (!(clip > 0.0f) || clip > 1.0f)) return SMOOTHROT_INVALID_ARG;
  if (K % (codes >= 16 ? 128 : 8) != 0 || K > kMaxWidth) return SMOOTHROT_UNSUPPORTED_K;
  if (M == 0) return SMOOTHROT_OK;
  if (M > 0x7fffffffLL / 2 || (Y_f16 == nullptr && H_f16 == nullptr)) return SMOOTHROT_INVALID_ARG;
  if (Y_f16 == nullptr && (post_norm || post_w != nullptr || gate != nullptr)) return SMOOTHROT_INVALID_ARG;
  if (post_w != nullptr && !post_norm) return SMOOTHROT_INVALID_ARG;
  if (H_out_f16 == nullptr && X_out_f16 == nullptr && codes == 0) return SMOOTHROT_INVALID_ARG;
  if (codes != 0 && (q_out == nullptr || (codes != 32) != (step_out != nullptr) || (codes >= 16 && scale_out == nullptr)))
    return SMOOTHROT_INVALID_ARG;
  if (H_out_f16 != nullptr && H_out_f16 == X_out_f16) return SMOOTHROT_INVALID_ARG;
  const struct { const void* p; int64_t ld; } rows[] = {{Y_f16, ldy}, {H_f16, ldh}, {H_out_f16, ldho}, {X_out_f16, ldxo}};
  for (const auto& r : rows)
    if (r.p != nullptr && r.ld < K) return SMOOTHROT_INVALID_ARG;
  for (const auto& r : rows)
    if (r.p != nullptr && (!aligned16(r.p) || r.ld % 8 != 0)) return SMOOTHROT_BAD_ALIGNMENT;
  for (const float* p : {post_w, gate, pre_w})
    if (p != nullptr && !aligned16(p)) return SMOOTHROT_BAD_ALIGNMENT;
  if (codes != 0 && (!aligned16(q_out) || (codes >= 16 && !aligned16(scale_out)))) return SMOOTHROT_BAD_ALIGNMENT;
  NormArgs a{};
  a.y = static_cast<const __half*>(Y_f16);
  a.h = static_cast<const __half*>(H_f16);
  a.ldy = ldy; a.ldh = ldh; a.ldho = ldho; a.ldxo = ldxo;
  a.rows = int(M);
  a.K = int(K);
  a.post_w = post_w; a.gate = gate; a.pre_w = pre_w;
  a.post_norm = post_norm;
  a.block_scale = block_scale; a.residual_scale = residual_scale;
  a.eps = double(eps);
  a.inv_k = 1.0 / double(K);
  a.h_out = static_cast<__half*>(H_out_f16);
  a.x_out = static_cast<__half*>(X_out_f16);
  a.clip = clip;
  a.q_out = q_out; a.scale_out = scale_out; a.step_out = step_out;
  const int chunks = int(K / 8);
  const int64_t sms = device_sm_count();
  const int ch = (M <= sms && chunks <= kMaxThreads) ? 1 : 4;
  const int T = ((chunks + ch - 1) / ch + 31) / 32 * 32;
  const int64_t cap = sms * (1024 / T > 0 ? 1024 / T : 1);
  const int64_t grid = M < cap ? M : cap;
  auto go = [&](auto kern) { return launch(kern, dim3(unsigned(grid)), T, 0, 0, static_cast<cudaStream_t>(stream), a); };
  switch (codes) {
    case 0: return ch == 1 ? go(add_norm_kernel<0, 1>) : go(add_norm_kernel<0, 4>);
    case 4: return ch == 1 ? go(add_norm_kernel<4, 1>) : go(add_norm_kernel<4, 4>);
    case 16: return ch == 1 ? go(add_norm_kernel<16, 1>) : go(add_norm_kernel<16, 4>);
    default: return ch == 1 ? go(add_norm_kernel<32, 1>) : go(add_norm_kernel<32, 4>);
  }
}

}  // extern "C"
