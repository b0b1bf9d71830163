// Microscaled 4-bit floating point: what its quantizers and products share.
//
// A code is e2m1 (sign, two bits of exponent, one of mantissa): 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
// negatives, two to a byte, the even position in bits 0-3.  Groups of 32 values have a scale that is a power of
// two (one byte, exponent + 127); groups of 16 an e4m3 scale and, above it, a step per row.
//
// Scales lie as the tensor core's scale copy wants them: 128 rows and 4 neighbouring groups are one block of 512
// bytes, row r at (r % 32) * 16 + (r / 32) * 4 with its 4 groups side by side; blocks follow one another along the
// row's groups, then along the rows.  The product reads whole blocks with one bulk copy and hands them on unchanged.
#pragma once

#include "common.cuh"
#include "rowquant.cuh"

namespace smoothrot {
namespace mx {

constexpr int kAtomRows = 128, kAtomGroups = 4, kAtomBytes = 512;

inline bool group_ok(int64_t group) { return group == 16 || group == 32; }

// Offset of the 4-byte word with the scales of groups 4 * quad .. 4 * quad + 3 of a row; quads = K / group / 4.
__host__ __device__ __forceinline__ int64_t scale_word(int64_t row, int quad, int quads) {
  return ((row >> 7) * quads + quad) * kAtomBytes + (row & 31) * 16 + ((row >> 5) & 3) * 4;
}

// Host: launches such a kernel, in clusters of `cluster` CTAs (0: as the kernel says).  A chain of short calls takes a
// microsecond less for each.
template <typename... Params, typename... Given>
inline int launch(void (*kern)(Params...), dim3 grid, int threads, int smem, int cluster, cudaStream_t stream, Given&&... given) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(unsigned(threads), 1, 1);
  cfg.dynamicSmemBytes = size_t(smem);
  cfg.stream = stream;
  cudaLaunchAttribute attrs[2] = {};
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = unsigned(cluster);
  attrs[1].val.clusterDim.y = 1;
  attrs[1].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = cluster > 0 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kern, given...) != cudaSuccess) {
    (void)cudaGetLastError();
    return SMOOTHROT_CUDA_ERROR;
  }
  count_launch();
  return launch_status();
}

// Kernels of this kind are launched so that one may be set up while the one before it in the stream finishes; each
// waits here, before it reads or writes what others may use.
// The wait comes first: a call that follows and waits for the end of this one has then waited for all before it too.
__device__ __forceinline__ void after_the_call_before() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Loads of what a call before may have written: volatile, so that none is moved to before that wait.  _once: data that is not read again.
__device__ __forceinline__ float load(const float* p) {
  float v;
  asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ float4 load(const float4* p) {
  float4 v;
  asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t load(const uint8_t* p) {
  uint32_t v;
  asm volatile("ld.global.u8 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load_once(const uint2* p) {
  uint2 v;
  asm volatile("ld.global.cs.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ uint4 load_once(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// ---- barriers of asynchronous copies ----

constexpr unsigned long long kWaitLimitNs = 2000000000ull;   // 2 s, of every wait
constexpr unsigned long long kDrainNs = 50000ull;            // pause before leaving after a timeout

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
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
__device__ __forceinline__ void drain() {
  const unsigned long long t0 = now_ns();
  while (now_ns() - t0 < kDrainNs) __nanosleep(1000);
}
// Host: reads a status word and, where asked, clears it.
inline int read_status_word(const int& symbol, int* out, int clear) {
  if (cudaMemcpyFromSymbol(out, symbol, sizeof(int)) != cudaSuccess) return SMOOTHROT_CUDA_ERROR;
  if (clear && *out != 0) {
    const int zero = 0;
    if (cudaMemcpyToSymbol(symbol, &zero, sizeof(int)) != cudaSuccess) return SMOOTHROT_CUDA_ERROR;
  }
  return SMOOTHROT_OK;
}

// Eight values to eight codes, round to nearest, ties to the even code, saturating at 6.
__device__ __forceinline__ uint32_t to_codes(const float (&q)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(r)
      : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
  return r;
}

// Group of 32: the scale's byte from the largest magnitude's bits.  The exponent E is the least one with
// max <= 7 * 2^E: a largest value above 6 * 2^E is then off by no more than the half of the code's widest
// gap (4 to 6), which a plain floor(log2 max) - 2 exceeds between 7 and 8.  A group with an infinity or NaN
// has the scale NaN, so that every product with it is NaN.
__device__ __forceinline__ uint32_t scale_byte_32(uint32_t top) {
  if (top == 0u) return 127u;
  if (top >= 0x7f800000u) return 255u;
  const int byte = int(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);   // 7 = 1.75 * 2^2
  return uint32_t(byte < 0 ? 0 : byte);
}
// 2^-(byte - 127), for bytes below 254
__device__ __forceinline__ float inverse_scale_32(uint32_t byte) { return __uint_as_float((254u - (byte & 255u)) << 23); }

// Groups of 16: the row's step from its largest magnitude's bits, the least power of two with max <= 2688 * step
// (2688 = 6 * 448, the largest code times the largest scale), 2^-100 at the least.  A power of two, so that every quotient below
// is as exact as a division by the scale's 4 bits.  1 for a row of zeros, NaN for one that holds an infinity or NaN.
__device__ __forceinline__ float row_step_16(uint32_t top) {
  if (top == 0u) return 1.0f;
  if (top >= 0x7f800000u) return __uint_as_float(0x7fffffffu);
  const int e = int(top >> 23) - 11 + ((top & 0x7fffffu) > 0x280000u ? 1 : 0);     // 2688 = 1.3125 * 2^11
  return __uint_as_float(uint32_t(e < 27 ? 27 : e) << 23);
}

// An e4m3 scale nearest to t >= 0, saturating at 448; its byte and its value.
__device__ __forceinline__ uint32_t to_e4m3(float t) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(t));
  return uint32_t(r) & 255u;
}
__device__ __forceinline__ float from_e4m3(uint32_t byte) {
  uint32_t h2;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"(uint16_t(byte)));
  return __half2float(__ushort_as_half(uint16_t(h2 & 0xffffu)));
}

// v / d as the correctly rounded quotient from the rounded reciprocal and one residual correction: values and scales
// of few bits meet the borders between codes all the time, where a quotient that is off by its last bit is another code.
__device__ __forceinline__ float quotient(float v, float d, float inv) {
  const float q = __fmul_rn(v, inv);
  return __fmaf_rn(__fmaf_rn(-q, d, v), inv, q);
}

// ---- rows: a thread holds 2 W neighbouring values of one, as W words of two fp16 values ----

template <int W>
struct Part {
  uint32_t w[W];
};
// A unit is 32 bytes.  `wide`: the address is a multiple of 32, as one load; otherwise two of 16 bytes.
constexpr int kUnit = 16;
typedef Part<kUnit / 2> Unit;

__device__ __forceinline__ Unit load_unit(const __half* p, bool wide) {
  Unit u;
  if (wide) {
    asm volatile("ld.global.cs.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(u.w[0]), "=r"(u.w[1]), "=r"(u.w[2]), "=r"(u.w[3]), "=r"(u.w[4]), "=r"(u.w[5]), "=r"(u.w[6]), "=r"(u.w[7])
                 : "l"(p));
  } else {
    const uint4 a = load_once(reinterpret_cast<const uint4*>(p)), b = load_once(reinterpret_cast<const uint4*>(p) + 1);
    u = Unit{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
  }
  return u;
}
__device__ __forceinline__ void store_unit(__half* p, const Unit& u, bool wide) {
  if (wide) {
    asm volatile("st.global.cs.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(u.w[0]), "r"(u.w[1]), "r"(u.w[2]),
                 "r"(u.w[3]), "r"(u.w[4]), "r"(u.w[5]), "r"(u.w[6]), "r"(u.w[7]));
  } else {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(u.w[0], u.w[1], u.w[2], u.w[3]));
    __stcs(reinterpret_cast<uint4*>(p) + 1, make_uint4(u.w[4], u.w[5], u.w[6], u.w[7]));
  }
}
inline bool wide_ok(const void* p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0 && ld % 16 == 0; }

template <int W>
__device__ __forceinline__ Part<W> no_values() {
  Part<W> u;
#pragma unroll
  for (int i = 0; i < W; ++i) u.w[i] = 0u;
  return u;
}
template <int W>
__device__ __forceinline__ void widen(const Part<W>& u, f32x2 (&v)[W]) {
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = half2_to_f32x2(u.w[i]);
}
template <int W>
__device__ __forceinline__ Part<W> narrow(const f32x2 (&v)[W]) {
  Part<W> u;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    float lo, hi;
    unpack2(v[i], lo, hi);
    const __half2 h = __floats2half2_rn(lo, hi);
    u.w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return u;
}

// Largest magnitude, as an fp32 value; a NaN wins over everything.
template <int W>
__device__ __forceinline__ float top_of(const Part<W>& u) {
  __half2 m[W];
#pragma unroll
  for (int i = 0; i < W; ++i) m[i] = __habs2(*reinterpret_cast<const __half2*>(&u.w[i]));
#pragma unroll
  for (int s = W / 2; s > 0; s /= 2)
#pragma unroll
    for (int i = 0; i < s; ++i) m[i] = __hmax2_nan(m[i], m[i + s]);
  return __half2float(__hmax_nan(__low2half(m[0]), __high2half(m[0])));
}
__device__ __forceinline__ float max_abs(float a, float b) {
  float r;
  asm("{\n\t.reg .f32 x, y;\n\tabs.f32 x, %1;\n\tabs.f32 y, %2;\n\tmax.NaN.f32 %0, x, y;\n\t}" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
template <int W>
__device__ __forceinline__ float top_of(const f32x2 (&v)[W]) {
  float m[W];
#pragma unroll
  for (int i = 0; i < W; ++i) {
    float a, b;
    unpack2(v[i], a, b);
    m[i] = max_abs(a, b);
  }
#pragma unroll
  for (int s = W / 2; s > 0; s /= 2)
#pragma unroll
    for (int i = 0; i < s; ++i) m[i] = max_abs(m[i], m[i + s]);
  return m[0];
}

// 1 / d by one step of Newton's iteration on the hardware's approximation: the correctly rounded reciprocal, compared with it for every
// mantissa, where it and d are normal numbers (steps from 2^-100 to 2^117).  The quantizer of 8192 x 4096: 18.4 -> 17.2 us.
__device__ __forceinline__ float reciprocal(float d) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
  return __fmaf_rn(r, __fmaf_rn(-d, r, 1.0f), r);
}

// A row's step as groups of 16 need it.
struct RowStep {
  float step, six, inverse;      // 6 step and its reciprocal
};
__device__ __forceinline__ RowStep row_step(float step) {
  const float six = __fmul_rn(6.0f, step);
  return RowStep{step, six, reciprocal(six)};
}
// A thread's values, with their largest magnitude, to codes (a word for every 8) and the scale byte of their group.  The threads
// of a group, neighbouring lanes, take part together.  ANY_STEP: the step is not the row's own, and values may be so far beyond it that
// no fp32 number holds the quotient.
template <int GROUP, bool ANY_STEP = false, int W>
__device__ __forceinline__ Part<W / 4> encode(const f32x2 (&v)[W], float top, const RowStep& row, uint32_t* byte) {
  uint32_t most = __float_as_uint(top);
#pragma unroll
  for (int x = 1; x < GROUP / (2 * W); x *= 2) most = max(most, __shfl_xor_sync(0xffffffffu, most, x));
  f32x2 q[W];
  if constexpr (GROUP == 32) {
    *byte = scale_byte_32(most);
    const float inv = inverse_scale_32(*byte);
    const f32x2 inv2 = pack2(inv, inv);
#pragma unroll
    for (int i = 0; i < W; ++i) q[i] = mul2(v[i], inv2);
  } else {
    const float t = __uint_as_float(most);
    // beyond the largest scale: that one, but the quotient of an infinity is NaN
    const bool beyond = t >= 448.0f * row.six;
    *byte = to_e4m3(beyond && most < 0x7f800000u ? 448.0f : quotient(t, row.six, row.inverse));
    const float d = __fmul_rn(from_e4m3(*byte), row.step);
    const float inv = d == 0.0f ? 0.0f : reciprocal(d);
    const f32x2 inv2 = pack2(inv, inv), neg2 = pack2(-d, -d);
#pragma unroll
    for (int i = 0; i < W; ++i) {      // quotient()
      const f32x2 r = mul2(v[i], inv2);
      q[i] = fma2(fma2(r, neg2, v[i]), inv2, r);
    }
    if (ANY_STEP && beyond) {      // rare: what is beyond 8 units is 6 of them as well
      const float far = 8.0f * d;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        float lo, hi;
        unpack2(v[i], lo, hi);
        q[i] = pack2(fabsf(lo) > far ? copysignf(8.0f, lo) : quotient(lo, d, inv), fabsf(hi) > far ? copysignf(8.0f, hi) : quotient(hi, d, inv));
      }
    }
  }
  Part<W / 4> codes;
#pragma unroll
  for (int c = 0; c < W / 4; ++c) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(q[4 * c + i], f[2 * i], f[2 * i + 1]);
    codes.w[c] = to_codes(f);
  }
  return codes;
}
// Offset within its row's scales of the scale byte of the part'th 2 W values, and whether their thread is the one of its group that
// writes it.  64 bits: beyond 2^29 values of a row in groups of 16 the offset passes 2^32.
template <int GROUP, int W>
__device__ __forceinline__ int64_t scale_offset(int part) {
  const int group = part / (GROUP / (2 * W));
  return int64_t(group >> 2) * kAtomBytes + (group & 3);
}
template <int GROUP, int W>
__device__ __forceinline__ bool writes_scale(int part) { return part % (GROUP / (2 * W)) == 0; }

// Walsh rotation of blocks of N = 32, 64 or 128 values over the lanes that hold them, 2 W values each; strides 1, 2, 4, ... in turn,
// then one product with 1 / sqrt(N).
template <int N, int W>
__device__ __forceinline__ void walsh_rows(f32x2 (&v)[W], float norm, int lane) {
#pragma unroll
  for (int i = 0; i < W; ++i) {
    float a, b;
    unpack2(v[i], a, b);
    v[i] = pack2(__fadd_rn(a, b), __fsub_rn(a, b));
  }
#pragma unroll
  for (int s = 1; s < W; s *= 2)
#pragma unroll
    for (int i = 0; i < W; ++i)
      if ((i & s) == 0) {
        const f32x2 a = v[i], b = v[i + s];
        v[i] = add2(a, b);
        v[i + s] = sub2(a, b);
      }
#pragma unroll
  for (int x = 1; x * 2 * W < N; x *= 2) {
    const float sign = (lane & x) ? -1.0f : 1.0f;
    const f32x2 sign2 = pack2(sign, sign);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const f32x2 p = __shfl_xor_sync(0xffffffffu, v[i], x);
      v[i] = fma2(sign2, v[i], p);       // p + v or p - v
    }
  }
  const f32x2 norm2 = pack2(norm, norm);
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = mul2(v[i], norm2);
}

// The sum of squares in 64 bits.  Statistics so good, rounded once, are the same fp32 number whatever the order of the
// additions, and codes of what is computed from them do not hang on it.
template <int W>
__device__ __forceinline__ double sum_of_squares(const Part<W>& u) {
  double s = 0.0, r = 0.0;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    double lo, hi;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f64.f16 %0, l;\n\tcvt.f64.f16 %1, h;\n\t}" : "=d"(lo), "=d"(hi) : "r"(u.w[i]));
    s = fma(lo, lo, s);
    r = fma(hi, hi, r);
  }
  return s + r;
}

}  // namespace mx
}  // namespace smoothrot
