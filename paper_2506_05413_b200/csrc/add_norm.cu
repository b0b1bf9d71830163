// The residual stream between two blocks: a block's output, normalised and gated, added to the stream, and the norm in
// front of the next block with that block's quantizer behind it.
//
//   z  = y                         or  y * rstd(y) * post_w
//   h' = fp16(residual_scale * h + block_scale * gate * z)
//   x  = fp16(h' * rstd(h') * pre_w)           rstd(r) = 1 / sqrt(mean(r^2) + eps)
//   x, and / or its codes: one step per row as in smoothrot_quant_act_plain, or microscaled as in smoothrot_mx_quant
//
// One pass: a row is read once (4 bytes a value), lives in registers as fp16 through both norms and leaves as h' and x
// or codes.  A CTA takes two rows at a time, so that it meets and fetches the weights half as often, a thread 16 neighbouring
// values of each.  Every product and sum of the formulas is rounded by itself and the norms' statistics are kept in 64
// bits and rounded once to fp32, so the results do not hang on how a row is shared out, and the codes are those of the
// quantizer run on x.
#include "mx.cuh"

namespace smoothrot {
namespace mx {

__device__ int g_norm_status = 0;
__device__ unsigned long long g_norm_wait_limit_ns = kWaitLimitNs;
constexpr int kNormRows = 51;      // code of a wait for rows that ran out

namespace {

constexpr int kMaxThreads = 1024;
constexpr int64_t kMaxWidth = 2 * kUnit * kMaxThreads;
constexpr int kRing = 3;           // pairs of rows that a CTA has in shared memory or on their way there

struct NormArgs {
  const __half *y, *h;
  int64_t ldy, ldh, ldho, ldxo;
  int rows, K;
  int units, half_unit;       // of a row; the one with 8 values, or -1
  bool wide;                  // every row starts on 32 bytes
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

// The last unit of a row whose length is not a multiple of 16 has 8 values.
__device__ __forceinline__ Unit load_part(const __half* p, bool wide, bool half) {
  if (!half) return load_unit(p, wide);
  return Unit{__ldcs(reinterpret_cast<const uint4*>(p)), make_uint4(0u, 0u, 0u, 0u)};
}
__device__ __forceinline__ void store_part(__half* p, const Unit& u, bool wide, bool half) {
  if (!half) store_unit(p, u, wide);
  else __stcs(reinterpret_cast<uint4*>(p), u.a);
}
// A unit's 16 weights.
__device__ __forceinline__ void load_weights(const float* w, int unit, bool half, f32x2 (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (!half || i < 2) f = __ldg(reinterpret_cast<const float4*>(w + unit * kUnit) + i);
    v[2 * i] = pack2(f.x, f.y);
    v[2 * i + 1] = pack2(f.z, f.w);
  }
}
__device__ __forceinline__ void times(f32x2 (&v)[8], const f32x2 (&w)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = mul2(v[i], w[i]);
}
__device__ __forceinline__ void times(f32x2 (&v)[8], float f) {
  const f32x2 f2 = pack2(f, f);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = mul2(v[i], f2);
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ bool wait_rows(uint32_t bar, uint32_t parity) {
  if (bar_try(bar, parity)) return true;
  const unsigned long long t0 = now_ns();
  while (!bar_try(bar, parity))
    if (now_ns() - t0 > g_norm_wait_limit_ns) {
      atomicCAS(&g_norm_status, 0, kNormRows);
      return false;
    }
  return true;
}
__device__ __forceinline__ Unit shared_unit(uint32_t addr, bool half) {
  Unit u = zero_unit();
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.a.x), "=r"(u.a.y), "=r"(u.a.z), "=r"(u.a.w) : "r"(addr) : "memory");
  if (!half)
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(u.b.x), "=r"(u.b.y), "=r"(u.b.z), "=r"(u.b.w) : "r"(addr + 16u) : "memory");
  return u;
}

// CODES: 0 none, 4 one step per row, 16 and 32 microscaled groups.  U units a thread, R rows at a time.  Where R is 2 the
// CTA comes back for more rows: they come through shared memory, two pairs ahead, and a thread keeps the weights of its unit in registers: read again for every row they took
// three times what the rows themselves took of the path to the registers (8192 rows of 4096: 106 us).
template <int CODES, int U, int R>
__global__ void __launch_bounds__(R == 2 ? 512 : kMaxThreads) add_norm_kernel(const NormArgs a) {
  __shared__ double sums[2][2][R][kMaxThreads / 32];
  __shared__ float tops[2][R][kMaxThreads / 32];
  const int t = threadIdx.x, T = blockDim.x, lane = t & 31, wid = t >> 5, warps = T >> 5;
  after_the_call_before();
  constexpr bool KEEP = R == 2;
  f32x2 kept[KEEP ? 3 : 1][8];
  if constexpr (KEEP) {
    if (t < a.units) {
      if (a.post_w != nullptr) load_weights(a.post_w, t, t == a.half_unit, kept[0]);
      if (a.gate != nullptr) load_weights(a.gate, t, t == a.half_unit, kept[1]);
      if (a.pre_w != nullptr) load_weights(a.pre_w, t, t == a.half_unit, kept[2]);
    }
  }
  auto weigh = [&](f32x2 (&v)[8], int which, const float* w, int unit, bool half) {
    if (w == nullptr) return;
    if constexpr (KEEP) {
      times(v, kept[which]);
    } else {
      load_weights(w, unit, half, kept[0]);
      times(v, kept[0]);
    }
  };
  // KEEP: a ring of row pairs, each [row][y, h][K]
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ __align__(8) unsigned long long bars[kRing];
  const uint32_t row_bytes = uint32_t(a.K) * 2u, ring_at = smem_u32(ring), bar_at = smem_u32(bars);
  auto fetch = [&](int m, int s) {      // by one thread
    const int rows = min(R, a.rows - m);
    bar_expect(bar_at + 8u * s, uint32_t(rows) * row_bytes * uint32_t((a.y != nullptr) + (a.h != nullptr)));
    for (int r = 0; r < rows; ++r) {
      const uint32_t dst = ring_at + uint32_t(s * R + r) * 2u * row_bytes;
      if (a.y != nullptr) bulk_load(dst, a.y + int64_t(m + r) * a.ldy, row_bytes, bar_at + 8u * s);
      if (a.h != nullptr) bulk_load(dst + row_bytes, a.h + int64_t(m + r) * a.ldh, row_bytes, bar_at + 8u * s);
    }
  };
  if (KEEP) {
    if (t == 0) {
      for (int s = 0; s < kRing; ++s) bar_init(bar_at + 8u * s, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      for (int s = 0; s < kRing; ++s)
        if (int64_t(blockIdx.x + s * gridDim.x) * R < a.rows) fetch(int(blockIdx.x + s * gridDim.x) * R, s);
    }
    __syncthreads();
  }
  const f32x2 one = pack2(1.0f, 1.0f);
  int stage = 0;
  uint32_t phase = 0;
  // what is kept for one pair of rows and the next are two sets in turn
  for (int m = blockIdx.x * R, parity = 0; m < a.rows; m += gridDim.x * R, parity ^= 1) {
    Unit y[R][U], h[R][U];
    bool there = true;
    if (KEEP) there = wait_rows(bar_at + 8u * stage, phase);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int unit = t + u * T;
        const bool on = unit < a.units && m + r < a.rows, half = unit == a.half_unit;
        if (KEEP) {
          const uint32_t at = ring_at + uint32_t(stage * R + r) * 2u * row_bytes + uint32_t(unit) * 32u;
          y[r][u] = on && a.y != nullptr ? shared_unit(at, half) : zero_unit();
          h[r][u] = on && a.h != nullptr ? shared_unit(at + row_bytes, half) : zero_unit();
        } else {
          y[r][u] = on && a.y != nullptr ? load_part(a.y + int64_t(m + r) * a.ldy + unit * kUnit, a.wide, half) : zero_unit();
          h[r][u] = on && a.h != nullptr ? load_part(a.h + int64_t(m + r) * a.ldh + unit * kUnit, a.wide, half) : zero_unit();
        }
      }
    if (KEEP) {
      if (__syncthreads_or(!there)) {       // a wait ran out: what is on its way lands before the memory is given back
        drain();
        return;
      }
      const int64_t next = int64_t(m) + int64_t(kRing) * gridDim.x * R;
      if (t == 0 && next < a.rows) fetch(int(next), stage);
      if (++stage == kRing) {
        stage = 0;
        phase ^= 1u;
      }
    }
    // v: a thread's part of each row's sum of squares; afterwards the rows' rstd
    auto statistics = [&](double (&v)[R], float (&rstd)[R], double (*slot)[kMaxThreads / 32]) {
      // with two rows, even lanes go on with the first and odd lanes with the second
      double mine = v[0];
      if (R == 2) mine = (lane & 1 ? v[R - 1] : v[0]) + __shfl_xor_sync(0xffffffffu, lane & 1 ? v[0] : v[R - 1], 1);
#pragma unroll
      for (int o = R; o < 32; o *= 2) mine += __shfl_xor_sync(0xffffffffu, mine, o);
      if (warps > 1) {
        if (lane < R) slot[lane][wid] = mine;
        __syncthreads();
        mine = lane / R < warps ? slot[lane % R][lane / R] : 0.0;
#pragma unroll
        for (int o = R; o < 32; o *= 2) mine += __shfl_xor_sync(0xffffffffu, mine, o);      // R == 2: at most 16 warps
      }
      const float f = rstd_of(mine, a.inv_k, a.eps);
#pragma unroll
      for (int r = 0; r < R; ++r) rstd[r] = __shfl_sync(0xffffffffu, f, r);
    };
    double sum[R];
    float rstd[R];
    if (a.post_norm) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        sum[r] = 0.0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          sum[r] += sum_of_squares(y[r][u]);
        }
      }
      statistics(sum, rstd, sums[parity][0]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      sum[r] = 0.0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int unit = t + u * T;
        if (unit >= a.units || m + r >= a.rows) continue;
        const bool half = unit == a.half_unit;
        f32x2 z[8], s[8];
        if (a.y != nullptr) {
          widen(y[r][u], z);
          if (a.post_norm) {
            times(z, rstd[r]);
            weigh(z, 0, a.post_w, unit, half);
          }
          weigh(z, 1, a.gate, unit, half);
          times(z, a.block_scale);
        }
        if (a.h != nullptr) {
          widen(h[r][u], s);
          if (a.residual_scale != 1.0f) times(s, a.residual_scale);
          if (a.y != nullptr) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = fma2(z[i], one, s[i]);      // a sum: a packed addition could take z's last product in
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) s[i] = z[i];
        }
        h[r][u] = narrow(s);
        if (a.h_out != nullptr) store_part(a.h_out + int64_t(m + r) * a.ldho + unit * kUnit, h[r][u], a.wide, half);
        sum[r] += sum_of_squares(h[r][u]);
      }
    }
    if (CODES == 0 && a.x_out == nullptr) continue;
    statistics(sum, rstd, sums[parity][1]);
    float top[R][U], most[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      most[r] = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int unit = t + u * T;
        const bool half = unit == a.half_unit;
        top[r][u] = 0.0f;
        if (unit >= a.units || m + r >= a.rows) continue;
        f32x2 x[8];
        widen(h[r][u], x);
        times(x, rstd[r]);
        weigh(x, 2, a.pre_w, unit, half);
        h[r][u] = narrow(x);
        if (a.x_out != nullptr) store_part(a.x_out + int64_t(m + r) * a.ldxo + unit * kUnit, h[r][u], a.wide, half);
        if constexpr (CODES != 0) top[r][u] = top_of(h[r][u]);
        most[r] = max_abs(most[r], top[r][u]);
      }
    }
    if constexpr (CODES != 0) {
      if constexpr (CODES == 4 || CODES == 16) {
  #pragma unroll
        for (int r = 0; r < R; ++r) {
          most[r] = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most[r])));
          if (lane == 0) tops[parity][r][wid] = most[r];
        }
        if (warps > 1) {
          __syncthreads();
  #pragma unroll
          for (int r = 0; r < R; ++r)
            most[r] = __uint_as_float(__reduce_max_sync(0xffffffffu, lane < warps ? __float_as_uint(tops[parity][r][lane]) : 0u));
        }
      }
  #pragma unroll
      for (int r = 0; r < R; ++r) {
        if (m + r >= a.rows) break;
        float step = 1.0f, inv = 0.0f;
        if constexpr (CODES == 4) {
          step = step_from_absmax(most[r], a.clip);
          inv = __frcp_rn(step);
          if (t == 0) a.step_out[m + r] = step;
        } else if constexpr (CODES == 16) {
          step = row_step_16(__float_as_uint(most[r]));
          if (t == 0) a.step_out[m + r] = step;
          if (!(step > 0.0f)) step = 1.0f;
        }
  #pragma unroll
        for (int u = 0; u < U; ++u) {
          const int unit = t + u * T;
          f32x2 x[8];
          widen(h[r][u], x);
          if constexpr (CODES == 4) {
            uint32_t word[2] = {0u, 0u};
  #pragma unroll
            for (int i = 0; i < 16; ++i) {
              float lo, hi;
              unpack2(x[i / 2], lo, hi);
              const float c = fmaxf(fminf(rintf(quotient(i % 2 ? hi : lo, step, inv)), 7.0f), -8.0f);
              word[i / 8] |= (uint32_t(int(c)) & 15u) << (4 * (i % 8));
            }
            uint32_t* to = reinterpret_cast<uint32_t*>(a.q_out + int64_t(m + r) * (a.K >> 1)) + 2 * unit;
            if (unit < a.units) {
              to[0] = word[0];
              if (unit != a.half_unit) to[1] = word[1];
            }
          } else if constexpr (CODES >= 16) {
            uint32_t byte;
            const uint2 codes = encode<CODES>(x, top[r][u], step, &byte);
            if (unit < a.units) {
              __stcs(reinterpret_cast<uint2*>(a.q_out) + int64_t(m + r) * a.units + unit, codes);
              if (writes_scale<CODES>(unit))
                a.scale_out[scale_word(m + r, 0, a.units / (CODES / 4)) + scale_offset<CODES>(unit)] = uint8_t(byte);
            }
          }
        }
      }
    }
  }
}

}  // namespace
}  // namespace mx
}  // namespace smoothrot

extern "C" {

int smoothrot_norm_status_word(int* out, int clear) {
  return smoothrot::mx::read_status_word(smoothrot::mx::g_norm_status, out, clear);
}

int smoothrot_norm_set_wait_limit_ns(uint64_t ns) {
  const unsigned long long v = ns == 0 ? smoothrot::mx::kWaitLimitNs : static_cast<unsigned long long>(ns);
  return cudaMemcpyToSymbol(smoothrot::mx::g_norm_wait_limit_ns, &v, sizeof(v)) == cudaSuccess ? SMOOTHROT_OK
                                                                                                 : SMOOTHROT_CUDA_ERROR;
}

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
  a.units = int((K + kUnit - 1) / kUnit);
  a.half_unit = K % kUnit != 0 ? a.units - 1 : -1;
  a.wide = true;
  for (const auto& r : rows) a.wide = a.wide && (r.p == nullptr || wide_ok(r.p, r.ld));
  const int per = a.units <= kMaxThreads ? 1 : 2;
  const int T = ((a.units + per - 1) / per + 31) / 32 * 32;
  const int64_t sms = device_sm_count();
  // two rows at a time where a row fits half the threads and there are rows for every place
  const bool two = T <= 512 && M > sms * (1024 / T);
  const int64_t blocks = two ? (M + 1) / 2 : M, places = two ? sms * (512 / T) : sms * (1024 / T);
  const dim3 grid(unsigned(blocks < places ? blocks : places));
  const int ring_bytes = int(kRing * 2 * 2 * K * 2);
  auto go = [&](auto one_unit, auto two_units, auto two_rows) {
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!two) return per == 1 ? launch(one_unit, grid, T, 0, 0, st, a) : launch(two_units, grid, T, 0, 0, st, a);
    if (!allow_dynamic_smem(reinterpret_cast<const void*>(two_rows), ring_bytes)) return int(SMOOTHROT_CUDA_ERROR);
    return launch(two_rows, grid, T, ring_bytes, 0, st, a);
  };
#define SR_NORM(C) go(add_norm_kernel<C, 1, 1>, add_norm_kernel<C, 2, 1>, add_norm_kernel<C, 1, 2>)
  switch (codes) {
    case 0: return SR_NORM(0);
    case 4: return SR_NORM(4);
    case 16: return SR_NORM(16);
    default: return SR_NORM(32);
  }
#undef SR_NORM
}

}  // extern "C"
