// Attention of one new token per sequence over the paged key-value cache (layout: paged.cuh).
//
//   y = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale q.k_j - m),   m the running maximum,
//
// in one pass over the cache: every warp takes every fourth token of its sequence and keeps its own
// maximum, sum and output; the four meet in shared memory.
#include "paged.cuh"

namespace smoothrot {
namespace paged {

__device__ int g_decode_status = 0;

constexpr int kDecodeWarps = 4;

struct DecodeArgs {
  const __half* q;
  int64_t ldq;
  const int32_t* table;     // [batch][max_pages]
  int64_t max_pages;
  const int32_t* lengths;
  __half* y;
  int64_t ldy;
  int n_heads;
  float scale;
};

template <int D, int kBits>
__device__ __forceinline__ void load_row(const void* cache, const float2* params, const Cache& c, int64_t page, int head,
                                         int offset, int lane, float (&x)[D / 32]) {
  const int64_t row = head_row(c, page, head, offset);
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const int at = i * 32 + lane;
    if (kBits == 16) {
      x[i] = __half2float(reinterpret_cast<const __half*>(cache)[row * D + at]);
    } else {
      const uint8_t byte = reinterpret_cast<const uint8_t*>(cache)[row * (D / 2) + at / 2];
      const float2 p = params[param_row(c, page, head * D / kGroup, offset)];
      x[i] = (float((byte >> (4 * (at & 1))) & 15) - p.y) * p.x;
    }
  }
}

template <int D, int kBits>
__global__ void __launch_bounds__(32 * kDecodeWarps)
attn_decode_kernel(DecodeArgs a, Cache c) {
  constexpr int R = D / 32;
  const int b = blockIdx.y, h = blockIdx.x;
  const int kv = h / (a.n_heads / c.kv_heads);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int64_t len = a.lengths[b];
  if (len < 0 || len > a.max_pages * c.page_size) {
    if (threadIdx.x == 0) atomicCAS(&g_decode_status, 0, int(kDecodeRange));
    len = len < 0 ? 0 : a.max_pages * c.page_size;
  }
  float q[R], o[R], m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    q[i] = __half2float(a.q[b * a.ldq + int64_t(h) * D + i * 32 + lane]) * a.scale;
    o[i] = 0.0f;
  }
  for (int64_t j = warp; j < len; j += kDecodeWarps) {
    const int64_t page = a.table[b * a.max_pages + (j >> c.page_shift)];
    if (page < 0 || page >= c.pages) {
      if (lane == 0) atomicCAS(&g_decode_status, 0, int(kDecodeRange));
      continue;
    }
    const int offset = int(j & (c.page_size - 1));
    float x[R];
    load_row<D, kBits>(c.k, c.k_params, c, page, kv, offset, lane, x);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < R; ++i) s += q[i] * x[i];
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) s += __shfl_xor_sync(0xffffffffu, s, k);
    const float top = fmaxf(m, s);
    const float base = top == -INFINITY ? 0.0f : top;
    const float keep = expf(m - base), p = expf(s - base);
    load_row<D, kBits>(c.v, c.v_params, c, page, kv, offset, lane, x);
#pragma unroll
    for (int i = 0; i < R; ++i) o[i] = o[i] * keep + p * x[i];
    l = l * keep + p;
    m = top;
  }
  __shared__ float so[kDecodeWarps][D], sm[kDecodeWarps], sl[kDecodeWarps];
#pragma unroll
  for (int i = 0; i < R; ++i) so[warp][i * 32 + lane] = o[i];
  if (lane == 0) {
    sm[warp] = m;
    sl[warp] = l;
  }
  __syncthreads();
  float top = -INFINITY;
  for (int w = 0; w < kDecodeWarps; ++w) top = fmaxf(top, sm[w]);
  const float base = top == -INFINITY ? 0.0f : top;
  float total = 0.0f;
  for (int w = 0; w < kDecodeWarps; ++w) total += sl[w] * expf(sm[w] - base);
  for (int d = threadIdx.x; d < D; d += blockDim.x) {
    float y = 0.0f;
    for (int w = 0; w < kDecodeWarps; ++w) y += so[w][d] * expf(sm[w] - base);
    a.y[b * a.ldy + int64_t(h) * D + d] = __float2half_rn(len == 0 ? 0.0f : y / total);
  }
}

}  // namespace paged
}  // namespace smoothrot

extern "C" {

int smoothrot_decode_status_word(int* out, int clear) {
  return smoothrot::paged::read_status_word(smoothrot::paged::g_decode_status, out, clear);
}

size_t smoothrot_attn_decode_workspace_bytes(int64_t B, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim) {
  (void)B; (void)n_heads; (void)n_kv_heads; (void)head_dim;
  return 0;
}

int smoothrot_attn_decode(const void* Q_f16, int64_t ldq, int64_t B, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                          int bits, int64_t pages, int64_t page_size, const void* k_cache, const void* v_cache,
                          const float* k_params, const float* v_params, const int32_t* block_table, int64_t max_pages,
                          const int32_t* lengths, float scale, void* Y_f16, int64_t ldy, void* workspace,
                          size_t workspace_bytes, void* stream) {
  using namespace smoothrot;
  using namespace smoothrot::paged;
  if (B < 0 || B > 8192 || n_heads <= 0 || n_heads > 65535 || max_pages < 0) return SMOOTHROT_INVALID_ARG;
  const int sizes = check_sizes(n_kv_heads, head_dim, bits, pages, page_size);
  if (sizes != SMOOTHROT_OK) return sizes;
  if (n_heads % n_kv_heads != 0 || max_pages * page_size > INT32_MAX || !(scale == scale)) return SMOOTHROT_INVALID_ARG;
  if (B == 0) return SMOOTHROT_OK;
  if (Q_f16 == nullptr || Y_f16 == nullptr || lengths == nullptr || ldq < n_heads * head_dim || ldy < n_heads * head_dim)
    return SMOOTHROT_INVALID_ARG;
  if (max_pages > 0 && block_table == nullptr) return SMOOTHROT_INVALID_ARG;
  if (pages > 0) {
    const int pointers = check_pointers(bits, k_cache, v_cache, k_params, v_params);
    if (pointers != SMOOTHROT_OK) return pointers;
  }
  if (!aligned16(Q_f16) || !aligned16(Y_f16) || ldq % 8 != 0 || ldy % 8 != 0) return SMOOTHROT_BAD_ALIGNMENT;
  if (workspace_bytes < smoothrot_attn_decode_workspace_bytes(B, n_heads, n_kv_heads, head_dim)) return SMOOTHROT_WORKSPACE_TOO_SMALL;
  (void)workspace;
  DecodeArgs a;
  a.q = static_cast<const __half*>(Q_f16); a.ldq = ldq;
  a.table = block_table; a.max_pages = max_pages; a.lengths = lengths;
  a.y = static_cast<__half*>(Y_f16); a.ldy = ldy;
  a.n_heads = int(n_heads); a.scale = scale;
  const Cache c = make_cache(n_kv_heads, head_dim, bits, pages, page_size, k_cache, v_cache, k_params, v_params);
  const dim3 grid{unsigned(n_heads), unsigned(B)};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (head_dim == 128) {
    if (bits == 16) attn_decode_kernel<128, 16><<<grid, 32 * kDecodeWarps, 0, st>>>(a, c);
    else attn_decode_kernel<128, 4><<<grid, 32 * kDecodeWarps, 0, st>>>(a, c);
  } else {
    if (bits == 16) attn_decode_kernel<64, 16><<<grid, 32 * kDecodeWarps, 0, st>>>(a, c);
    else attn_decode_kernel<64, 4><<<grid, 32 * kDecodeWarps, 0, st>>>(a, c);
  }
  count_launch();
  return launch_status();
}

}  // extern "C"
