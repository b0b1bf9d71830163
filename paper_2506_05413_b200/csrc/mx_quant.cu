// Quantizer of microscaled 4-bit floating point, with the layer's diagonal and a Walsh rotation in blocks on the way,
// and its inverse.  Formulas in mx.cuh and smoothrot.h.
//
// Streaming work: 2 bytes in, half a byte and a scale out per value, and bound by the instructions it issues rather than by
// memory unless they are few: a thread takes 16 neighbouring values at a time (one load of 32 bytes), so a group is one thread's or
// two neighbours', and keeps to its place in the rows, so that its part of the diagonal stays in registers and every offset
// but the row's is computed once.  Groups of 32 need nothing of the rest of their row: the rows are one long line of units,
// shared out evenly, and where they are rotated a thread takes 32 values, so that a block of 32 is its own and larger ones
// cross fewer lanes.  Groups of 16 have a step above them: a CTA takes two rows at a time and meets once for their maxima.
#include "mx.cuh"

namespace smoothrot {
namespace mx {
namespace {

constexpr int kMaxThreads = 1024;
constexpr int64_t kMaxWidth = 2 * kUnit * kMaxThreads;
constexpr int kFlatThreads = 256;

struct QuantArgs {
  const __half* x;
  int64_t ld;
  int rows, K;
  bool wide;
  const float* pre;
  float norm;
  uint8_t *q_out, *scale_out;
  float* step_out;
};

// The part'th 2 W values of a row, or of the diagonal
template <int W>
__device__ __forceinline__ Part<W> load_part(const __half* p, bool wide) {
  Part<W> u;
#pragma unroll
  for (int i = 0; i < W; i += 8) {
    const Unit h = load_unit(p + 2 * i, wide);
#pragma unroll
    for (int j = 0; j < 8; ++j) u.w[i + j] = h.w[j];
  }
  return u;
}
template <int W>
__device__ __forceinline__ void load_diagonal(const float* pre, int part, f32x2 (&d)[W]) {
#pragma unroll
  for (int i = 0; i < W / 2; ++i) {
    const float4 w = load(reinterpret_cast<const float4*>(pre + part * 2 * W) + i);
    d[2 * i] = pack2(w.x, w.y);
    d[2 * i + 1] = pack2(w.z, w.w);
  }
}
// Values with the diagonal and the rotation, and their largest magnitude.
template <int WALSH, bool PRE, int W>
__device__ __forceinline__ float transform(const Part<W>& raw, const f32x2 (&diagonal)[W], float norm, int lane, f32x2 (&v)[W]) {
  widen(raw, v);
  if constexpr (!PRE && WALSH == 0) return top_of(raw);
  if constexpr (PRE) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = mul2(v[i], diagonal[i]);
  }
  if constexpr (WALSH != 0) walsh_rows<WALSH>(v, norm, lane);
  return top_of(v);
}
template <int GROUP, int W>
__device__ __forceinline__ void put(const QuantArgs& a, int m, int part, uint32_t offset, const Part<W / 4>& codes, uint32_t byte) {
  uint8_t* to = a.q_out + int64_t(m) * (a.K / 2) + part * W;
  if constexpr (W == 16) __stcs(reinterpret_cast<uint4*>(to), make_uint4(codes.w[0], codes.w[1], codes.w[2], codes.w[3]));
  else __stcs(reinterpret_cast<uint2*>(to), make_uint2(codes.w[0], codes.w[1]));
  if (writes_scale<GROUP, W>(part)) a.scale_out[scale_word(m, 0, a.K / (4 * GROUP)) + offset] = uint8_t(byte);
}

// Groups of 32: `lines` rows side by side are under way, a thread takes its 2 W values of every lines-th row.  8192 x 4096: 14.9 us
// (5.7 TB/s, 0.87 of the copy rate), rotated in blocks of 32 16.9, of 64 19.5, of 128 with a diagonal 23.8 (3.6 TB/s): issue, and shuffles.
__host__ __device__ constexpr int flat_words(int walsh) { return walsh != 0 ? 16 : 8; }

template <int WALSH, bool PRE>
__global__ void __launch_bounds__(kFlatThreads, WALSH != 0 && PRE ? 2 : WALSH != 0 ? 3 : 4) mx_quant32_kernel(const QuantArgs a, const int lines) {
  constexpr int W = flat_words(WALSH);
  const int lane = threadIdx.x & 31, parts = a.K / (2 * W);
  const int64_t i = int64_t(blockIdx.x) * kFlatThreads + threadIdx.x;
  const int line = int(i / parts), part = int(i - int64_t(line) * parts);
  const bool on = line < lines;         // lanes of a rotation block or a group are on or off together
  const uint32_t offset = uint32_t(scale_offset<32, W>(part));      // rows end at kMaxWidth
  f32x2 diagonal[W];
  after_the_call_before();
  if (PRE && on) load_diagonal(a.pre, part, diagonal);
  const __half* src = a.x + int64_t(line) * a.ld + part * 2 * W;
  const int64_t stride = int64_t(lines) * a.ld;
  constexpr int R = 2;
  for (int m = line; m - line < a.rows; m += R * lines, src += R * stride) {
    Part<W> raw[R];
#pragma unroll
    for (int r = 0; r < R; ++r) raw[r] = on && m + r * lines < a.rows ? load_part<W>(src + r * stride, a.wide) : no_values<W>();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      f32x2 v[W];
      const float top = transform<WALSH, PRE>(raw[r], diagonal, a.norm, lane, v);
      uint32_t byte;
      const Part<W / 4> codes = encode<32>(v, top, RowStep{}, &byte);
      if (on && m + r * lines < a.rows) put<32, W>(a, m + r * lines, part, offset, codes, byte);
    }
  }
}

// Groups of 16: U times 2 W values a thread (the second ones a row's length of threads further), R rows at a time.  8192 x 4096: 17.2 us
// (4.9 TB/s), with a diagonal 22.8 (it spills 18 registers), with that and blocks of 128 29.0: issue (two thirds of the slots).  32 values
// a thread without a rotation: 19.5 to 21; with a diagonal 21.9, 1 to 14 % faster at seven of ten sizes, but 300 x 4096 3.3 -> 4.5 and 1000 x
// 2048 3.5 -> 4.8.
__host__ __device__ constexpr int row_threads(int walsh) { return walsh != 0 ? 512 : 1024; }

template <int WALSH, bool PRE, int U>
__global__ void __launch_bounds__(row_threads(WALSH)) mx_quant16_kernel(const QuantArgs a) {
  constexpr int W = flat_words(WALSH), R = U == 1 && WALSH == 0 ? 2 : 1;
  __shared__ float red[2][R][kMaxThreads / 32];
  const int t = threadIdx.x, T = blockDim.x, lane = t & 31, warps = T >> 5, parts = a.K / (2 * W);
  f32x2 diagonal[W];
  after_the_call_before();
  if (PRE && U == 1 && t < parts) load_diagonal(a.pre, t, diagonal);
  Part<W> raw[R][U];
  auto fetch = [&](int m) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int part = t + u * T;
        raw[r][u] = part < parts && m + r < a.rows ? load_part<W>(a.x + int64_t(m + r) * a.ld + part * 2 * W, a.wide) : no_values<W>();
      }
  };
  if (U == 1) fetch(blockIdx.x * R);
  for (int m = blockIdx.x * R, parity = 0; m < a.rows; m += gridDim.x * R, parity ^= 1) {
    if (U > 1) fetch(m);
    f32x2 v[R][U][W];
    float top[R][U], most[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      most[r] = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (PRE && U > 1 && t + u * T < parts) load_diagonal(a.pre, t + u * T, diagonal);
        top[r][u] = transform<WALSH, PRE>(raw[r][u], diagonal, a.norm, lane, v[r][u]);
        if (t + u * T >= parts) top[r][u] = 0.0f;
        most[r] = max_abs(most[r], top[r][u]);
      }
      most[r] = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most[r])));
      // two sets of words in turn: a warp that is ahead writes the other one
      if (lane == 0 && warps > 1) red[parity][r][t >> 5] = most[r];
    }
    if (U == 1) fetch(m + gridDim.x * R);      // on its way while these are coded
    if (warps > 1) __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (m + r >= a.rows) break;
      uint32_t bits = __float_as_uint(most[r]);
      if (warps > 1) bits = __reduce_max_sync(0xffffffffu, lane < warps ? __float_as_uint(red[parity][r][lane]) : 0u);
      float step = row_step_16(bits);
      if (t == 0) a.step_out[m + r] = step;
      if (!(step > 0.0f)) step = 1.0f;      // NaN: whatever the codes are, the row's values are NaN
      const RowStep row = row_step(step);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int part = t + u * T;
        if constexpr (W == 8) {
          uint32_t byte;
          const Part<2> codes = encode<16>(v[r][u], top[r][u], row, &byte);
          if (part < parts) put<16, 8>(a, m + r, part, uint32_t(scale_offset<16, 8>(part)), codes, byte);
        } else {
          // two groups of 16, each as the other kind of thread would have it
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            f32x2 half[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) half[i] = v[r][u][8 * g + i];
            uint32_t byte;
            const Part<2> codes = encode<16>(half, top_of(half), row, &byte);
            if (part < parts) put<16, 8>(a, m + r, 2 * part + g, uint32_t(scale_offset<16, 8>(2 * part + g)), codes, byte);
          }
        }
      }
    }
  }
}

// A word's eight codes as four pairs of fp16 values, exact.
__device__ __forceinline__ uint4 from_codes(uint32_t word) {
  uint4 h;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(h.x), "=r"(h.y), "=r"(h.z), "=r"(h.w)
      : "r"(word));
  return h;
}

// As mx_quant32_kernel: a thread keeps to its unit of every lines-th row.  8192 x 4096: 15.3 us in groups of 32, 16.4 of 16 (5.5, 5.2 TB/s).
template <int GROUP>
__global__ void __launch_bounds__(kFlatThreads)
mx_dequant_kernel(const uint8_t* q, const uint8_t* scale, const float* step, int rows, int units, int lines, __half* y, int64_t ldy,
                  bool wide) {
  const int64_t i = int64_t(blockIdx.x) * kFlatThreads + threadIdx.x;
  const int line = int(i / units), unit = int(i - int64_t(line) * units);
  if (line >= lines) return;
  const int64_t offset = scale_offset<GROUP, 8>(unit);
  after_the_call_before();
  constexpr int R = 4;
  for (int m = line; m < rows; m += R * lines) {
    uint2 word[R];
    uint32_t byte[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = min(m + r * lines, rows - 1);
      word[r] = load_once(reinterpret_cast<const uint2*>(q) + int64_t(row) * units + unit);
      byte[r] = load(scale + scale_word(row, 0, units / (GROUP / 4)) + offset);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = m + r * lines;
      if (row >= rows) break;
      float d = GROUP == 16 ? from_e4m3(byte[r])
                            : __uint_as_float(byte[r] == 0u ? 0x00400000u : byte[r] == 255u ? 0x7fffffffu : byte[r] << 23);
      if (step != nullptr) d = __fmul_rn(d, load(step + row));
      const uint4 lo = from_codes(word[r].x), hi = from_codes(word[r].y);
      const Unit codes{{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}};
      f32x2 v[8];
      widen(codes, v);
      const f32x2 d2 = pack2(d, d);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = mul2(v[k], d2);
      store_unit(y + int64_t(row) * ldy + unit * kUnit, narrow(v), wide);
    }
  }
}

// Rows side by side for a kernel that shares out units: as many as give every SM `threads` threads, fewer where the last
// round of rows would be thin.
int lines_for(int64_t rows, int64_t parts, int64_t threads) {
  int64_t lines = device_sm_count() * threads / parts;
  if (lines < 1) lines = 1;
  if (lines > rows) lines = rows;
  const int64_t rounds = (rows + lines - 1) / lines;
  return int((rows + rounds - 1) / rounds);
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
  QuantArgs a{};
  a.x = static_cast<const __half*>(X_f16);
  a.ld = ldx;
  a.rows = int(M);
  a.K = int(K);
  a.wide = wide_ok(X_f16, ldx);
  a.pre = pre;
  a.norm = walsh != 0 ? float(1.0 / sqrt(double(walsh))) : 1.0f;
  a.q_out = q_out;
  a.scale_out = scale_out;
  a.step_out = step_out;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (group == 32) {
    const int64_t parts = K / (2 * flat_words(walsh));
    const int lines = lines_for(M, parts, walsh == 0 ? 1024 : pre == nullptr ? 768 : 512);
    const dim3 grid(unsigned((lines * parts + kFlatThreads - 1) / kFlatThreads));
    auto go = [&](auto kern) { return launch(kern, grid, kFlatThreads, 0, 0, st, a, lines); };
    switch (walsh) {
      case 0: return pre ? go(mx_quant32_kernel<0, true>) : go(mx_quant32_kernel<0, false>);
      case 32: return pre ? go(mx_quant32_kernel<32, true>) : go(mx_quant32_kernel<32, false>);
      case 64: return pre ? go(mx_quant32_kernel<64, true>) : go(mx_quant32_kernel<64, false>);
      default: return pre ? go(mx_quant32_kernel<128, true>) : go(mx_quant32_kernel<128, false>);
    }
  }
  const int parts = int(K / (2 * flat_words(walsh))), most = row_threads(walsh), per = parts <= most ? 1 : 2;
  const int T = ((parts + per - 1) / per + 31) / 32 * 32;
  const int64_t rows_each = per == 1 && walsh == 0 ? 2 : 1, blocks = (M + rows_each - 1) / rows_each;
  const int64_t cap = int64_t(device_sm_count()) * (most / T);
  const dim3 grid(unsigned(blocks < cap ? blocks : cap));
  auto go = [&](auto one, auto two) { return per == 1 ? launch(one, grid, T, 0, 0, st, a) : launch(two, grid, T, 0, 0, st, a); };
#define SR_QUANT16(W) (pre ? go(mx_quant16_kernel<W, true, 1>, mx_quant16_kernel<W, true, 2>) \
                           : go(mx_quant16_kernel<W, false, 1>, mx_quant16_kernel<W, false, 2>))
  switch (walsh) {
    case 0: return SR_QUANT16(0);
    case 32: return SR_QUANT16(32);
    case 64: return SR_QUANT16(64);
    default: return SR_QUANT16(128);
  }
#undef SR_QUANT16
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
  const int units = int(K / kUnit), lines = lines_for(M, units, 2048);
  const dim3 grid(unsigned((int64_t(lines) * units + kFlatThreads - 1) / kFlatThreads));
  auto go = [&](auto kern) {
    return launch(kern, grid, kFlatThreads, 0, 0, static_cast<cudaStream_t>(stream), q, scale, step, int(M), units, lines,
                  static_cast<__half*>(Y_f16), ldy, wide_ok(Y_f16, ldy));
  };
  return group == 32 ? go(mx_dequant_kernel<32>) : go(mx_dequant_kernel<16>);
}

}  // extern "C"
