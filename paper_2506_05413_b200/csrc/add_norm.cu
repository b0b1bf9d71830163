// The residual stream between two blocks: a block's output, normalised and gated, added to the stream, and the norm in
// front of the next block with that block's quantizer behind it.
//
//   z  = y                         or  y * rstd(y) * post_w
//   h' = fp16(residual_scale * h + block_scale * gate * z)
//   x  = fp16(h' * rstd(h') * pre_w)           rstd(r) = 1 / sqrt(mean(r^2) + eps)
//   x, and / or its codes: one step per row as in smoothrot_quant_act_plain, or microscaled as in smoothrot_mx_quant
//
// One pass: a row is read once (4 bytes a value), lives in registers as fp16 through both norms and leaves as h' and x
// or codes, a thread holding 8 or 16 neighbouring values.  Every product and sum of the formulas is rounded by itself and the norms'
// statistics are kept in 64 bits and rounded once to fp32, so the results do not hang on how a row is shared out, and the codes
// are those of the quantizer run on x.
//
// With many rows it is bound by the instructions that takes and, more, by the exchanges between a row's threads that the statistics
// need (with 256 threads to a row of 4096 values those took 18 of 60 us).  So a row is one team's of few threads, up to 64 values each,
// which meet cheaply and have several chains of instructions side by side; teams fill an SM independently of one another and share the
// weights in its shared memory; rows come through shared memory too, the next one while the last is worked on.
#include "mx.cuh"

namespace smoothrot {
namespace mx {

__device__ int g_norm_status = 0;
__device__ unsigned long long g_norm_wait_limit_ns = kWaitLimitNs;
constexpr int kNormRows = 51;      // code of a wait for rows that ran out, in the test probe too

namespace {

constexpr int kMaxThreads = 1024;
constexpr int kChunk = 8;                            // values of a thread
constexpr int kMostChunks = 4;                       // of a thread, in long rows
constexpr int64_t kMaxWidth = kChunk * kMostChunks * kMaxThreads;
constexpr int kTeamThreads = 512;                    // of a CTA of teams: 128 registers each
constexpr int kMaxTeams = 15;                        // a barrier each
typedef Part<kChunk / 2> Chunk;

struct NormArgs {
  const __half *y, *h;
  int64_t ldy, ldh, ldho, ldxo;
  int rows, K;
  int chunks;                 // of a row
  bool wide;                  // rows of h_out and x_out start on 32 bytes
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

__device__ __forceinline__ Chunk load_chunk(const __half* p) {
  const uint4 a = load_once(reinterpret_cast<const uint4*>(p));
  return Chunk{{a.x, a.y, a.z, a.w}};
}
__device__ __forceinline__ Unit shared_unit(const uint8_t* p) {
  const uint4 a = *reinterpret_cast<const uint4*>(p), b = *reinterpret_cast<const uint4*>(p + 16);
  return Unit{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ void store_chunk(__half* p, const Chunk& u) {
  __stcs(reinterpret_cast<uint4*>(p), make_uint4(u.w[0], u.w[1], u.w[2], u.w[3]));
}
// The weights of the part'th 2 W values; null: ones, which change nothing.
template <int W>
__device__ __forceinline__ void load_weights(const float* w, int part, f32x2 (&v)[W]) {
#pragma unroll
  for (int i = 0; i < W / 2; ++i) {
    const float4 f = w != nullptr ? load(reinterpret_cast<const float4*>(w + part * 2 * W) + i) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
    v[2 * i] = pack2(f.x, f.y);
    v[2 * i + 1] = pack2(f.z, f.w);
  }
}
template <int W>
__device__ __forceinline__ void times(f32x2 (&v)[W], const f32x2 (&w)[W]) {
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = mul2(v[i], w[i]);
}
template <int W>
__device__ __forceinline__ void times(f32x2 (&v)[W], float f) {
  const f32x2 f2 = pack2(f, f);
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = mul2(v[i], f2);
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

// The threads that share a row: `warps` warps, which meet at barrier `id`; `slot` is their first place of those for a value per warp.
struct Team {
  int id, warps, slot;
  __device__ __forceinline__ void meet() const { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(warps * 32) : "memory"); }
};

// Whether a wait of one of the team's threads ran out: one answer for all.  They leave then, once what is on its way has landed and the
// memory may be given back.
__device__ __forceinline__ bool team_gives_up(bool there, const Team& team, int threads) {
  uint32_t late;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(late) : "r"(uint32_t(!there)), "r"(team.id), "r"(threads) : "memory");
  if (late != 0) drain();
  return late != 0;
}

// rstd of a row from its threads' parts of the sum of squares.
__device__ __forceinline__ float statistics(double mine, double* slots, const Team& team, int wid, const NormArgs& a) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o /= 2) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  if (team.warps > 1) {
    double* slot = slots + team.slot;
    if (lane == 0) slot[wid] = mine;
    team.meet();
    if (team.warps <= 4) {
      mine = slot[0] + slot[1];
      if (team.warps > 2) mine += slot[2] + (team.warps > 3 ? slot[3] : 0.0);
    } else {
      mine = lane < team.warps ? slot[lane] : 0.0;
#pragma unroll
      for (int o = 16; o > 0; o /= 2) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    }
  }
  return rstd_of(mine, a.inv_k, a.eps);
}
// The largest of a row's threads' values.
__device__ __forceinline__ float largest(float mine, float* slots, const Team& team, int wid) {
  const int lane = threadIdx.x & 31;
  uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(mine));
  if (team.warps > 1) {
    if (lane == 0) slots[team.slot + wid] = __uint_as_float(m);
    team.meet();
    m = __reduce_max_sync(0xffffffffu, lane < team.warps ? __float_as_uint(slots[team.slot + lane]) : 0u);
  }
  return __uint_as_float(m);
}

// z (the block's output as it came) into the stream: fp16(residual_scale * h + block_scale * gate * z).
template <bool POST, int W>
__device__ __forceinline__ Part<W> add(const Part<W>& y, const Part<W>& h, float rstd, const f32x2 (&post)[W], const f32x2 (&gate)[W],
                                       const NormArgs& a) {
  f32x2 z[W], s[W];
  widen(y, z);
  if constexpr (POST) {
    times(z, rstd);
    times(z, post);
  }
  times(z, gate);
  times(z, a.block_scale);
  widen(h, s);
  times(s, a.residual_scale);
  const f32x2 one = pack2(1.0f, 1.0f);
#pragma unroll
  for (int i = 0; i < W; ++i) s[i] = fma2(z[i], one, s[i]);      // a sum: a packed addition could take a product before it in
  return narrow(s);
}
template <int W>
__device__ __forceinline__ Part<W> norm(const Part<W>& h, float rstd, const f32x2 (&pre)[W]) {
  f32x2 x[W];
  widen(h, x);
  times(x, rstd);
  times(x, pre);
  return narrow(x);
}
// Codes of a thread's values; every thread of the warp takes part, `on` ones write.
template <int CODES, int W>
__device__ __forceinline__ void put_codes(const Part<W>& x16, float top, const RowStep& row, int m, int part, bool on, const NormArgs& a) {
  f32x2 x[W];
  widen(x16, x);
  Part<W / 4> codes;
  uint32_t byte = 0;
  if constexpr (CODES == 4) {
    // quotient(), two at a time; added to 1.5 * 2^23 it is rounded to the integer, ties to even, whose low bits are the code
    const float magic = 12582912.0f;
    const f32x2 inv2 = pack2(row.inverse, row.inverse), neg2 = pack2(-row.step, -row.step), magic2 = pack2(magic, magic);
#pragma unroll
    for (int c = 0; c < W / 4; ++c) {
      codes.w[c] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 r = mul2(x[4 * c + i], inv2);
        const f32x2 q = fma2(fma2(r, neg2, x[4 * c + i]), inv2, r);
        float lo, hi;
        unpack2(add2(q, magic2), lo, hi);
        lo = fmaxf(fminf(lo, magic + 7.0f), magic - 8.0f);
        hi = fmaxf(fminf(hi, magic + 7.0f), magic - 8.0f);
        const uint32_t pair = (__float_as_uint(lo) & 15u) | ((__float_as_uint(hi) & 15u) << 4);
        codes.w[c] |= pair << (8 * i);
      }
    }
  } else {
    codes = encode<CODES>(x, top, row, &byte);
  }
  if (!on) return;
  uint32_t* to = reinterpret_cast<uint32_t*>(a.q_out + int64_t(m) * (a.K >> 1)) + part * (W / 4);
  if constexpr (W == 8) __stcs(reinterpret_cast<uint2*>(to), make_uint2(codes.w[0], codes.w[1]));
  else __stcs(to, codes.w[0]);
  if constexpr (CODES != 4)
    if (writes_scale<CODES, W>(part))
      a.scale_out[scale_word(m, 0, a.K / (4 * CODES)) + scale_offset<CODES, W>(part)] = uint8_t(byte);
}
// The step of a row from its largest magnitude, written by one thread.
template <int CODES>
__device__ __forceinline__ RowStep step_of(float most, int m, bool write, const NormArgs& a) {
  const float step = CODES == 4 ? step_from_absmax(most, a.clip) : row_step_16(__float_as_uint(most));
  if (write) a.step_out[m] = step;
  if (CODES == 4) return RowStep{step, 0.0f, __frcp_rn(step)};
  return row_step(step > 0.0f ? step : 1.0f);       // NaN: whatever the codes are, the row's values are NaN
}

// CODES: 0 none, 4 one step per row, 16 and 32 microscaled groups.  POST: a norm after the block.

// Weights in shared memory: values 4 i .. 4 i + 3 of unit u are float4 number i * units + u, so that a warp reads them without conflicts.
__device__ __forceinline__ void shared_weights(const float4* w, int unit, int units, f32x2 (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 f = w[i * units + unit];
    v[2 * i] = pack2(f.x, f.y);
    v[2 * i + 1] = pack2(f.z, f.w);
  }
}

// Many rows of up to 8192 values, whole units of 16, y and h both there: a team of `threads` threads takes a row, U units a
// thread.  Threads past a row's end take its last unit again, so that there is one course of instructions; they write nothing.
// 8192 x 4096 into codes: 41 us (5.3 TB/s), of groups of 16 45, integer ones 45, with a norm after the block 49 (4.5), 51 and 51, fp16 47
// (5.7).  Two exchanges of a row stand in line with its arithmetic at 16 warps an SM; issue (53 %) and the statistics in 64 bits (34 % of
// their pipe) alone do not bound it.
template <int CODES, bool POST, int U>
__global__ void __launch_bounds__(kTeamThreads) add_norm_teams_kernel(const NormArgs a, const int threads) {
  __shared__ double sums[2][2][kTeamThreads / 32];          // [row in turn][norm]: a warp that is ahead writes the other row's
  __shared__ float tops[2][kTeamThreads / 32];
  __shared__ __align__(8) unsigned long long bars[kMaxTeams];
  extern __shared__ __align__(128) uint8_t dynamic[];       // three arrays of weights, then each team's row [y, h][K]
  const int which = int(threadIdx.x) / threads, teams = int(blockDim.x) / threads;
  const Team team{1 + which, threads >> 5, which * (threads >> 5)};
  const int t = int(threadIdx.x) - which * threads, wid = t >> 5, units = a.K / kUnit;
  const uint32_t row_bytes = uint32_t(a.K) * 2u;
  float4* weights = reinterpret_cast<float4*>(dynamic);     // three times K / 4
  const uint8_t* rows = dynamic + size_t(a.K) * 12u + size_t(which) * 2u * row_bytes;
  const uint32_t row_at = smem_u32(rows), bar = smem_u32(bars) + 8u * which;
  auto fetch = [&](int64_t m) {      // by one thread
    bar_expect(bar, 2u * row_bytes);
    bulk_load(row_at, a.y + m * a.ldy, row_bytes, bar);
    bulk_load(row_at + row_bytes, a.h + m * a.ldh, row_bytes, bar);
  };
  int unit[U];
  bool on[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    unit[u] = min(t + u * threads, units - 1);
    on[u] = t + u * threads < units;
  }
  const int64_t first = int64_t(blockIdx.x) * teams + which, stride = int64_t(gridDim.x) * teams;
  after_the_call_before();
  if (t == 0) {
    bar_init(bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (first < a.rows) fetch(first);
  }
  const float* arrays[3] = {a.post_w, a.gate, a.pre_w};
#pragma unroll
  for (int w = POST ? 0 : 1; w < 3; ++w)
    for (int i = threadIdx.x; i < a.K / 4; i += blockDim.x) {
      // none: ones, which change nothing
      const float4 f = arrays[w] != nullptr ? load(reinterpret_cast<const float4*>(arrays[w]) + i) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
      weights[w * (a.K / 4) + (i & 3) * units + (i >> 2)] = f;
    }
  __syncthreads();
  int parity = 0;
  for (int64_t row = first; row < a.rows; row += stride, parity ^= 1) {
    const int m = int(row);
    Unit y[U], h[U];
    const bool there = wait_rows(bar, uint32_t(parity));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      y[u] = shared_unit(rows + unit[u] * 32);
      h[u] = shared_unit(rows + row_bytes + unit[u] * 32);
    }
    if (team_gives_up(there, team, threads)) return;
    if (t == 0 && row + stride < a.rows) fetch(row + stride);
    double sum = 0.0;
    float rstd = 1.0f;
    if constexpr (POST) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const double s = sum_of_squares(y[u]);
        sum += on[u] ? s : 0.0;
      }
      rstd = statistics(sum, sums[parity][0], team, wid, a);
      sum = 0.0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      f32x2 post[8], gate[8];
      if constexpr (POST) shared_weights(weights, unit[u], units, post);
      shared_weights(weights + a.K / 4, unit[u], units, gate);
      h[u] = add<POST>(y[u], h[u], rstd, post, gate, a);
      const double s = sum_of_squares(h[u]);
      sum += on[u] ? s : 0.0;
      if (a.h_out != nullptr && on[u]) store_unit(a.h_out + row * a.ldho + unit[u] * kUnit, h[u], a.wide);
    }
    if (CODES == 0 && a.x_out == nullptr) continue;
    rstd = statistics(sum, sums[parity][1], team, wid, a);
    float top[U], most = 0.0f;
    RowStep step{};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      f32x2 pre[8];
      shared_weights(weights + a.K / 2, unit[u], units, pre);
      h[u] = norm(h[u], rstd, pre);
      if (a.x_out != nullptr && on[u]) store_unit(a.x_out + row * a.ldxo + unit[u] * kUnit, h[u], a.wide);
      if constexpr (CODES != 0) {
        top[u] = top_of(h[u]);
        most = max_abs(most, top[u]);
      }
    }
    if constexpr (CODES != 0) {
      if constexpr (CODES != 32) step = step_of<CODES>(largest(most, tops[parity], team, wid), m, t == 0, a);
#pragma unroll
      for (int u = 0; u < U; ++u) put_codes<CODES>(h[u], top[u], step, m, unit[u], on[u], a);
    }
  }
}

// Few rows, long ones, or only one of y and h: a row at a time, U chunks a thread, straight from global memory.  1 x 4096: 2.5 us.  Many
// rows come to it where they are long or one-sided, and it is far from their bytes then: 4096 x 16384 into codes 105 us, with a norm after
// the block 157 (67 at the copy rate), 8192 x 4096 of the stream alone 70 (13).
template <int CODES, int U>
__global__ void __launch_bounds__(kMaxThreads) add_norm_kernel(const NormArgs a) {
  __shared__ double sums[2][2][kMaxThreads / 32];
  __shared__ float tops[2][kMaxThreads / 32];
  const int t = threadIdx.x, T = blockDim.x, wid = t >> 5;
  const Team team{1, T >> 5, 0};
  after_the_call_before();
  int parity = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, parity ^= 1) {
    const int m = int(row);
    Chunk y[U], h[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int chunk = t + u * T;
      const bool on = chunk < a.chunks;
      y[u] = on && a.y != nullptr ? load_chunk(a.y + row * a.ldy + chunk * kChunk) : no_values<4>();
      h[u] = on && a.h != nullptr ? load_chunk(a.h + row * a.ldh + chunk * kChunk) : no_values<4>();
    }
    double sum = 0.0;
    float rstd = 1.0f;
    if (a.post_norm) {
#pragma unroll
      for (int u = 0; u < U; ++u) sum += sum_of_squares(y[u]);
      rstd = statistics(sum, sums[parity][0], team, wid, a);
    }
    sum = 0.0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int chunk = t + u * T;
      if (chunk >= a.chunks) continue;
      if (a.y != nullptr) {
        f32x2 post[4], gate[4];
        load_weights(a.gate, chunk, gate);
        if (a.post_norm) load_weights(a.post_w, chunk, post);
        if (a.h == nullptr) {      // without the stream: nothing is added, a negative zero stays one
          f32x2 z[4];
          widen(y[u], z);
          if (a.post_norm) {
            times(z, rstd);
            times(z, post);
          }
          times(z, gate);
          times(z, a.block_scale);
          h[u] = narrow(z);
        } else {
          h[u] = a.post_norm ? add<true>(y[u], h[u], rstd, post, gate, a) : add<false>(y[u], h[u], rstd, gate, gate, a);
        }
      } else {
        f32x2 s[4];
        widen(h[u], s);
        times(s, a.residual_scale);
        h[u] = narrow(s);
      }
      if (a.h_out != nullptr) store_chunk(a.h_out + row * a.ldho + chunk * kChunk, h[u]);
      sum += sum_of_squares(h[u]);
    }
    if (CODES == 0 && a.x_out == nullptr) continue;
    rstd = statistics(sum, sums[parity][1], team, wid, a);
    float top[U], most = 0.0f;
    RowStep step{};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int chunk = t + u * T;
      top[u] = 0.0f;
      if (chunk >= a.chunks) continue;
      f32x2 pre[4];
      load_weights(a.pre_w, chunk, pre);
      h[u] = norm(h[u], rstd, pre);
      if (a.x_out != nullptr) store_chunk(a.x_out + row * a.ldxo + chunk * kChunk, h[u]);
      if constexpr (CODES != 0) top[u] = top_of(h[u]);
      most = max_abs(most, top[u]);
    }
    if constexpr (CODES != 0) {
      if constexpr (CODES != 32) step = step_of<CODES>(largest(most, tops[parity], team, wid), m, t == 0, a);
#pragma unroll
      for (int u = 0; u < U; ++u) put_codes<CODES>(h[u], top[u], step, m, t + u * T, t + u * T < a.chunks, a);
    }
  }
}

// Test probe: a team waits for rows that nobody sends, and leaves as the kernel's teams do.
constexpr int kProbeThreads = 64;
__global__ void norm_wait_probe_kernel() {
  __shared__ __align__(8) unsigned long long storage;
  const uint32_t bar = smem_u32(&storage);
  if (threadIdx.x == 0) {
    bar_init(bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  (void)team_gives_up(wait_rows(bar, 0u), Team{1, kProbeThreads / 32, 0}, kProbeThreads);
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

int smoothrot_debug_norm_wait_expiry(void* stream) {
  smoothrot::mx::norm_wait_probe_kernel<<<1, smoothrot::mx::kProbeThreads, 0, static_cast<cudaStream_t>(stream)>>>();
  smoothrot::count_launch();
  return smoothrot::launch_status();
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
  if ((codes == 0 && (q_out != nullptr || step_out != nullptr)) || (codes < 16 && scale_out != nullptr)) return SMOOTHROT_INVALID_ARG;
  if (H_out_f16 != nullptr && H_out_f16 == X_out_f16) return SMOOTHROT_INVALID_ARG;
  const struct { const void* p; int64_t ld; } rows[] = {{Y_f16, ldy}, {H_f16, ldh}, {H_out_f16, ldho}, {X_out_f16, ldxo}};
  for (const auto& r : rows)
    if (r.p != nullptr && r.ld < K) return SMOOTHROT_INVALID_ARG;
  for (const auto& r : rows)
    if (r.p != nullptr && (!aligned16(r.p) || r.ld % 8 != 0)) return SMOOTHROT_BAD_ALIGNMENT;
  for (const float* p : {post_w, gate, pre_w})
    if (p != nullptr && !aligned16(p)) return SMOOTHROT_BAD_ALIGNMENT;
  if (codes != 0 && (!aligned16(q_out) || (codes >= 16 && !aligned16(scale_out)))) return SMOOTHROT_BAD_ALIGNMENT;
  // written over an input: row for row, or one row's output would be another's input
  for (int i = 0; i < 2; ++i)
    for (int o = 2; o < 4; ++o)
      if (M > 1 && rows[i].p != nullptr && rows[i].p == rows[o].p && rows[i].ld != rows[o].ld) return SMOOTHROT_INVALID_ARG;
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
  a.chunks = int(K / kChunk);
  const int64_t sms = device_sm_count();
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  // A row at a time while there is a place for each.  Beyond, teams whose threads take 1, 2 or 4 units: more of them let more rows be under
  // way and cost a round of rows more.  An estimate in us decides: a fixed part, which grows with the weights, and a time per round of rows,
  // less where a round leaves threads over.  Measured, a row at a time | 1 | 2 | 4 units, with a norm after the block: 600 x 4096 11.7 |
  // 12.2 | 12.9 | 12.5, 2048 x 4096 32.0 | 22.6 | 21.3 | 21.1, 8192 x 4096 97 | 72 | 56 | 49; without: 7.9 | 8.4 | 9.2 | 10.0,
  // 22.1 | 15.8 | 15.1 | 17.7, 82 | 51 | 41 | 45.
  const int row_threads = (a.chunks + 31) / 32 * 32, units = int(K / kUnit);
  const bool may_team = K % kUnit == 0 && K <= 8192 && a.y != nullptr && a.h != nullptr;
  const int64_t at_once = may_team ? sms * (kMaxThreads / row_threads) : 0;
  const double thousands = double(K) / 1024.0;
  auto share = [](double used) { return 0.4 + 0.6 * used; };      // of a full round's time
  bool in_teams = false;
  int each = 0, T = 0, teams = 0;
  if (may_team && M > at_once) {
    const double f = share(double(kMaxThreads / row_threads * row_threads) / kMaxThreads), x = double(M) / double(at_once);
    double least = post_norm ? 4.0 + 4.0 * f * x : 2.0 + 2.9 * f * x;
    for (int e = 1, i = 0; e <= 4; e *= 2, ++i) {
      const int threads = ((units + e - 1) / e + 31) / 32 * 32, most = kTeamThreads / threads, n = most < kMaxTeams ? most : kMaxTeams;
      const double rounds = double((M + sms * n - 1) / (sms * n)), used = double(n * units) / double(kTeamThreads * e);
      const double fixed[2][3] = {{3.0, 3.0, 3.5}, {3.5, 4.3, 6.0}}, weights[2][3] = {{0.2, 0.2, 0.7}, {0.35, 0.35, 0.8}};
      const double round[2][3] = {{1.65, 2.7, 5.6}, {2.1 + 0.06 * thousands, 3.1 + 0.12 * thousands, 5.8}};
      const double us = fixed[post_norm][i] + weights[post_norm][i] * thousands + round[post_norm][i] * share(used) * rounds;
      if (us >= least) continue;
      least = us;
      in_teams = true;
      each = e;
      T = threads;
      teams = n;
    }
  }
  a.wide = (H_out_f16 == nullptr || wide_ok(H_out_f16, ldho)) && (X_out_f16 == nullptr || wide_ok(X_out_f16, ldxo));
  auto go_teams = [&](auto one, auto two, auto four) {
    const int bytes = int(3 * 4 * K + int64_t(teams) * 2 * 2 * K);
    const int64_t blocks = (M + teams - 1) / teams;
    const dim3 grid(unsigned(blocks < sms ? blocks : sms));
    auto kern = each == 1 ? one : each == 2 ? two : four;
    if (!allow_dynamic_smem(reinterpret_cast<const void*>(kern), bytes)) return int(SMOOTHROT_CUDA_ERROR);
    return launch(kern, grid, teams * T, bytes, 0, st, a, T);
  };
  const int per = a.chunks <= kMaxThreads ? 1 : a.chunks <= 2 * kMaxThreads ? 2 : kMostChunks;
  auto go_rows = [&](auto one, auto two, auto most) {
    const int threads = ((a.chunks + per - 1) / per + 31) / 32 * 32;
    const int64_t places = sms * (kMaxThreads / threads);
    const dim3 grid(unsigned(M < places ? M : places));
    return per == 1 ? launch(one, grid, threads, 0, 0, st, a)
                    : per == 2 ? launch(two, grid, threads, 0, 0, st, a) : launch(most, grid, threads, 0, 0, st, a);
  };
#define SR_TEAMS(C, P) go_teams(add_norm_teams_kernel<C, P, 1>, add_norm_teams_kernel<C, P, 2>, add_norm_teams_kernel<C, P, 4>)
#define SR_NORM(C)                                                                                                      \
  in_teams ? (post_norm ? SR_TEAMS(C, true) : SR_TEAMS(C, false))                                                       \
           : go_rows(add_norm_kernel<C, 1>, add_norm_kernel<C, 2>, add_norm_kernel<C, kMostChunks>)
  switch (codes) {
    case 0: return SR_NORM(0);
    case 4: return SR_NORM(4);
    case 16: return SR_NORM(16);
    default: return SR_NORM(32);
  }
#undef SR_NORM
#undef SR_TEAMS
}

}  // extern "C"
