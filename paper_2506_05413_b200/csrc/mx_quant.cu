// Quantizer of microscaled 4-bit floating point, with the layer's diagonal and a Walsh rotation in blocks on the way,
// and its inverse.  Formulas in mx.cuh and smoothrot.h.
//
// Streaming work: 2 bytes in, half a byte and a scale out per value.  A CTA takes a row at a time, a thread
// up to 4 chunks of 8 neighbouring values (16-byte loads, chunk c of thread t is chunk t + c T of the row), whose 8 codes are one
// aligned word of the output; groups, rotation blocks and the 4 scales that lie side by side are all made of the chunks
// of neighbouring lanes, so everything but a row's maximum (groups of 16 have a step above them) stays inside a warp.
// The next row's loads are in flight during the arithmetic.
#include "mx.cuh"

namespace smoothrot {
namespace mx {
namespace {

constexpr int kMaxThreads = 1024;
constexpr int64_t kMaxWidth = 8 * 4 * kMaxThreads;

template <int GROUP, int CH>
__global__ void __launch_bounds__(kMaxThreads)
mx_quant_kernel(const __half* __restrict__ x, int64_t ld, int rows, int K, const float* __restrict__ pre, int walsh,
                float norm, uint8_t* __restrict__ q_out, uint8_t* __restrict__ scale_out, float* __restrict__ step_out) {
  __shared__ uint32_t red[2][kMaxThreads / 32];
  const int t = threadIdx.x, T = blockDim.x, lane = t & 31;
  const int chunks = K >> 3, quads = K / (4 * GROUP);
  uint4 raw[CH];
  int m = blockIdx.x;
  after_the_call_before();
  if (m < rows) {
    const uint4* src = reinterpret_cast<const uint4*>(x + int64_t(m) * ld);
#pragma unroll
    for (int c = 0; c < CH; ++c) raw[c] = t + c * T < chunks ? __ldcs(src + t + c * T) : make_uint4(0u, 0u, 0u, 0u);
  }
  int parity = 0;
  for (; m < rows; m += gridDim.x, parity ^= 1) {
    float v[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      unpack2(half2_to_f32x2(raw[c].x), v[c][0], v[c][1]);
      unpack2(half2_to_f32x2(raw[c].y), v[c][2], v[c][3]);
      unpack2(half2_to_f32x2(raw[c].z), v[c][4], v[c][5]);
      unpack2(half2_to_f32x2(raw[c].w), v[c][6], v[c][7]);
    }
    const int next = m + gridDim.x;
    if (next < rows) {
      const uint4* src = reinterpret_cast<const uint4*>(x + int64_t(next) * ld);
#pragma unroll
      for (int c = 0; c < CH; ++c) raw[c] = t + c * T < chunks ? __ldcs(src + t + c * T) : make_uint4(0u, 0u, 0u, 0u);
    }
    if (pre != nullptr) {
      const float4* p = reinterpret_cast<const float4*>(pre);
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (t + c * T < chunks) {
          const float4 a = __ldg(p + 2 * (t + c * T)), b = __ldg(p + 2 * (t + c * T) + 1);
          const float d[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
          for (int i = 0; i < 8; ++i) v[c][i] = __fmul_rn(v[c][i], d[i]);
        }
    }
    if (walsh != 0) {
#pragma unroll
      for (int c = 0; c < CH; ++c) walsh_lanes(v[c], walsh, norm, lane);
    }
    float step = 1.0f;
    if constexpr (GROUP == 16) {
      uint32_t top = 0;
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, abs_bits(v[c][i]));
      top = __reduce_max_sync(0xffffffffu, top);
      if (T > 32) {
        // two sets of words in turn: a warp that is ahead writes the other one
        if (lane == 0) red[parity][t >> 5] = top;
        __syncthreads();
        top = __reduce_max_sync(0xffffffffu, lane < (T >> 5) ? red[parity][lane] : 0u);
      }
      step = row_step_16(top);
      if (t == 0) step_out[m] = step;
      if (!(step > 0.0f)) step = 1.0f;      // NaN: whatever the codes are, the row's values are NaN
    }
    uint32_t* q_row = reinterpret_cast<uint32_t*>(q_out + int64_t(m) * (K >> 1));
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int chunk = t + c * T;
      uint32_t byte;
      const uint32_t codes = GROUP == 32 ? encode_32(v[c], &byte) : encode_16(v[c], step, &byte);
      const uint32_t word = scale_quad<GROUP>(byte, lane);
      if (chunk < chunks) {
        __stcs(q_row + chunk, codes);
        if ((lane & (GROUP / 2 - 1)) == 0)
          *reinterpret_cast<uint32_t*>(scale_out + scale_word(m, chunk / (GROUP / 2), quads)) = word;
      }
    }
  }
}

// Four codes' values (a 16-bit part of a word) as four floats.
__device__ __forceinline__ void from_codes(uint32_t word, float (&v)[8]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(word));
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack2(half2_to_f32x2(h[i]), v[2 * i], v[2 * i + 1]);
}

// A thread per 8 values.
template <int GROUP>
__global__ void __launch_bounds__(256)
mx_dequant_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scale, const float* __restrict__ step,
                  int64_t total, int chunks, __half* __restrict__ y, int64_t ldy) {
  const int quads = chunks / (GROUP / 2);
  after_the_call_before();
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
    const int64_t m = i / chunks;
    const int chunk = int(i - m * chunks), group = chunk / (GROUP / 8);
    const uint32_t word = __ldcs(reinterpret_cast<const uint32_t*>(q) + i);
    const uint32_t byte = scale[scale_word(m, group >> 2, quads) + (group & 3)];
    float d = GROUP == 16 ? from_e4m3(byte)
                          : __uint_as_float(byte == 0u ? 0x00400000u : byte == 255u ? 0x7fffffffu : byte << 23);
    if (step != nullptr) d = __fmul_rn(d, __ldg(step + m));
    float v[8];
    from_codes(word, v);
    uint4 out;
    __half2* h = reinterpret_cast<__half2*>(&out);
#pragma unroll
    for (int k = 0; k < 4; ++k) h[k] = __floats2half2_rn(__fmul_rn(v[2 * k], d), __fmul_rn(v[2 * k + 1], d));
    __stcs(reinterpret_cast<uint4*>(y + m * ldy) + chunk, out);
  }
}

}  // namespace
}  // namespace mx
}  // namespace smoothrot

extern "C" {

size_t smoothrot_mx_scale_bytes(int64_t rows, int64_t K, int64_t group) {
  using namespace smoothrot::mx;
  if (rows <= 0 || K <= 0 || K % 128 != 0 || !group_ok(group)) return 0;
  return size_t((rows + kAtomRows - 1) / kAtomRows) * size_t(K / group / kAtomGroups) * kAtomBytes;
}

int smoothrot_mx_quant(const void* X_f16, int64_t M, int64_t K, int64_t ldx, int64_t group, const float* pre, int walsh,
                       uint8_t* q_out, uint8_t* scale_out, float* step_out, void* stream) {
  using namespace smoothrot;
  using namespace smoothrot::mx;
  if (M < 0 || K <= 0 || !group_ok(group)) return SMOOTHROT_INVALID_ARG;
  if (walsh != 0 && walsh != 32 && walsh != 64 && walsh != 128) return SMOOTHROT_INVALID_ARG;
  if (K % 128 != 0 || K > kMaxWidth) return SMOOTHROT_UNSUPPORTED_K;
  if (M == 0) return SMOOTHROT_OK;
  if (X_f16 == nullptr || q_out == nullptr || scale_out == nullptr || (group == 16) != (step_out != nullptr) || ldx < K ||
      M > 0x7fffffffLL / 2)
    return SMOOTHROT_INVALID_ARG;
  if (!aligned16(X_f16) || ldx % 8 != 0 || !aligned16(q_out) || !aligned16(scale_out) || (pre != nullptr && !aligned16(pre)))
    return SMOOTHROT_BAD_ALIGNMENT;
  const int chunks = int(K / 8);
  // one chunk a thread while the rows do not fill the machine (a row is then one load deep), four beyond
  const int64_t sms = device_sm_count();
  const int ch = (M <= sms && chunks <= kMaxThreads) ? 1 : 4;
  const int T = ((chunks + ch - 1) / ch + 31) / 32 * 32;
  const int64_t cap = sms * (1024 / T > 0 ? 1024 / T : 1);
  const int64_t grid = M < cap ? M : cap;
  const float norm = walsh != 0 ? float(1.0 / sqrt(double(walsh))) : 1.0f;
  auto go = [&](auto kern) {
    return launch(kern, dim3(unsigned(grid)), T, 0, 0, static_cast<cudaStream_t>(stream), static_cast<const __half*>(X_f16), ldx,
                  int(M), int(K), pre, walsh, norm, q_out, scale_out, step_out);
  };
  if (group == 32) return ch == 1 ? go(mx_quant_kernel<32, 1>) : go(mx_quant_kernel<32, 4>);
  return ch == 1 ? go(mx_quant_kernel<16, 1>) : go(mx_quant_kernel<16, 4>);
}

int smoothrot_mx_dequant(const uint8_t* q, const uint8_t* scale, const float* step, int64_t M, int64_t K, int64_t group,
                         void* Y_f16, int64_t ldy, void* stream) {
  using namespace smoothrot;
  using namespace smoothrot::mx;
  if (M < 0 || K <= 0 || !group_ok(group)) return SMOOTHROT_INVALID_ARG;
  if (K % 128 != 0 || K > (int64_t(1) << 30)) return SMOOTHROT_UNSUPPORTED_K;
  if (M == 0) return SMOOTHROT_OK;
  if (q == nullptr || scale == nullptr || Y_f16 == nullptr || ldy < K || M > 0x7fffffffLL / 2) return SMOOTHROT_INVALID_ARG;
  if (!aligned16(q) || !aligned16(scale) || !aligned16(Y_f16) || ldy % 8 != 0) return SMOOTHROT_BAD_ALIGNMENT;
  const int64_t total = M * (K / 8), blocks = (total + 255) / 256, cap = int64_t(device_sm_count()) * 32;
  auto go = [&](auto kern) {
    return launch(kern, dim3(unsigned(blocks < cap ? blocks : cap)), 256, 0, 0, static_cast<cudaStream_t>(stream), q, scale, step,
                  total, int(K / 8), static_cast<__half*>(Y_f16), ldy);
  };
  return group == 32 ? go(mx_dequant_kernel<32>) : go(mx_dequant_kernel<16>);
}

}  // extern "C"
