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

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Kernels of this kind are launched so that one may be set up while the one before it in the stream finishes; each
// waits here, before it reads or writes what others may use.
// The wait comes first: a call that follows and waits for the end of this one has then waited for all before it too.
__device__ __forceinline__ void after_the_call_before() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
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

// A thread's eight neighbouring values of a row to a word of codes.  The lanes of a warp hold neighbouring
// chunks of eight; all 32 take part, those past the row's end with zeros.
// GROUP 32: returns the scale byte of the thread's group.
__device__ __forceinline__ uint32_t encode_32(const float (&v)[8], uint32_t* byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, abs_bits(v[i]));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  *byte = scale_byte_32(top);
  const float inv = inverse_scale_32(*byte);
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = __fmul_rn(v[i], inv);
  return to_codes(q);
}
// GROUP 16, `step` the row's (any positive number where the caller gives it).
__device__ __forceinline__ uint32_t encode_16(const float (&v)[8], float step, uint32_t* byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, abs_bits(v[i]));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  *byte = to_e4m3(__fdiv_rn(__uint_as_float(top), __fmul_rn(6.0f, step)));
  const float d = __fmul_rn(from_e4m3(*byte), step);
  const float inv = d == 0.0f ? 0.0f : __frcp_rn(d);
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = quotient(v[i], d, inv);
  return to_codes(q);
}

// The scale bytes of 4 neighbouring groups as one word, in the first of their lanes (of every 16 lanes with groups
// of 32, of every 8 with groups of 16).
template <int GROUP>
__device__ __forceinline__ uint32_t scale_quad(uint32_t byte, int lane) {
  constexpr int per = GROUP / 8;      // lanes of a group
  uint32_t w = byte << (8 * ((lane / per) & 3));
  w |= __shfl_xor_sync(0xffffffffu, w, per);
  w |= __shfl_xor_sync(0xffffffffu, w, 2 * per);
  return w;
}

// Walsh rotation of blocks of n = 32, 64 or 128 neighbouring values, eight to a lane; strides 1, 2, 4, ... in turn, then
// one product with 1 / sqrt(n).
__device__ __forceinline__ void walsh_lanes(float (&v)[8], int n, float norm, int lane) {
#pragma unroll
  for (int s = 1; s < 8; s *= 2)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((i & s) == 0) {
        const float a = v[i], b = v[i + s];
        v[i] = __fadd_rn(a, b);
        v[i + s] = __fsub_rn(a, b);
      }
  for (int x = 1; 8 * x < n; x *= 2) {
    const float sign = (lane & x) ? -1.0f : 1.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __fmaf_rn(sign, v[i], __shfl_xor_sync(0xffffffffu, v[i], x));   // p + v or p - v
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], norm);
}

// Sums of squares of fp16 values as a pair of floats (sum and what its roundings left), two lanes of each at a time: a square
// of 11 bits is exact in fp32 and the error of every addition is kept, so the sum is good to some 2^-45.  The norm that
// follows is then the same fp32 number whatever the order of the additions, and codes of its results do not hang on it.
struct SquareSum {
  f32x2 s, e;
  __device__ __forceinline__ void clear() { s = pack2(0.0f, 0.0f); e = s; }
  __device__ __forceinline__ void add(f32x2 x) {
    const f32x2 p = mul2(x, x);
    const f32x2 t = add2(s, p);
    const f32x2 b = sub2(t, s);
    e = add2(e, add2(sub2(p, b), sub2(s, sub2(t, b))));
    s = t;
  }
  __device__ __forceinline__ double total() const {
    float a, b, c, d;
    unpack2(s, a, b);
    unpack2(e, c, d);
    return (double(a) + double(b)) + (double(c) + double(d));
  }
};

}  // namespace mx
}  // namespace smoothrot
