// Attention over packed prompts of different lengths: queries [total_q] and keys [total_k] of all sequences one after
// another, grouped heads, causal (aligned at the sequences' ends) or not.
//
//   y_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i.k_j - m_i),  j <= i + keys - queries where causal
//
// One warp per query row and head, one pass over the visible keys with a running maximum and sum.
#include "common.cuh"

namespace smoothrot {
namespace prefill {

__device__ int g_prefill_status = 0;
constexpr int kRange = 35;
constexpr int kWarps = 4;

struct Args {
  const __half *q, *k, *v;
  int64_t ldq, ldk, ldv, ldy;
  __half* y;
  int64_t total_q, total_k;
  const int32_t *cu_q, *cu_k;
  int batch, n_heads, group, causal;
  float scale;
};

template <int D>
__global__ void __launch_bounds__(32 * kWarps)
attn_prefill_kernel(Args a) {
  constexpr int R = D / 32;
  const int lane = threadIdx.x & 31;
  const int h = blockIdx.y, kv = h / a.group;
  for (int64_t i = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5); i < a.total_q; i += int64_t(gridDim.x) * kWarps) {
    int lo = 0, hi = a.batch;                 // the sequence b with cu_q[b] <= i < cu_q[b + 1]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.cu_q[mid] <= i) lo = mid; else hi = mid;
    }
    const int64_t q0 = a.cu_q[lo], q1 = a.cu_q[lo + 1], k0 = a.cu_k[lo], k1 = a.cu_k[lo + 1];
    if (i < q0 || i >= q1) continue;          // a row of no sequence
    if (q1 > a.total_q || k0 < 0 || k1 < k0 || k1 > a.total_k) {
      if (lane == 0) atomicCAS(&g_prefill_status, 0, kRange);
      continue;
    }
    int64_t seen = k1 - k0;
    if (a.causal) {
      const int64_t most = i - q0 + 1 + (k1 - k0) - (q1 - q0);
      seen = seen < most ? seen : most;
    }
    float q[R], o[R], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      q[r] = __half2float(a.q[i * a.ldq + int64_t(h) * D + r * 32 + lane]) * a.scale;
      o[r] = 0.0f;
    }
    for (int64_t j = k0; j < k0 + seen; ++j) {
      float s = 0.0f;
#pragma unroll
      for (int r = 0; r < R; ++r) s += q[r] * __half2float(a.k[j * a.ldk + int64_t(kv) * D + r * 32 + lane]);
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
      const float top = fmaxf(m, s);
      const float base = top == -INFINITY ? 0.0f : top;
      const float keep = expf(m - base), p = expf(s - base);
#pragma unroll
      for (int r = 0; r < R; ++r) o[r] = o[r] * keep + p * __half2float(a.v[j * a.ldv + int64_t(kv) * D + r * 32 + lane]);
      l = l * keep + p;
      m = top;
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      a.y[i * a.ldy + int64_t(h) * D + r * 32 + lane] = __float2half_rn(seen <= 0 ? 0.0f : o[r] / l);
  }
}

}  // namespace prefill
}  // namespace smoothrot

extern "C" {

int smoothrot_prefill_status_word(int* out, int clear) {
  if (cudaMemcpyFromSymbol(out, smoothrot::prefill::g_prefill_status, sizeof(int)) != cudaSuccess) return SMOOTHROT_CUDA_ERROR;
  if (clear && *out != 0) {
    const int zero = 0;
    if (cudaMemcpyToSymbol(smoothrot::prefill::g_prefill_status, &zero, sizeof(int)) != cudaSuccess) return SMOOTHROT_CUDA_ERROR;
  }
  return SMOOTHROT_OK;
}

int smoothrot_attn_prefill(const void* Q_f16, int64_t ldq, int64_t total_q, const void* K_f16, int64_t ldk, const void* V_f16,
                           int64_t ldv, int64_t total_k, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                           const int32_t* cu_q, const int32_t* cu_k, int64_t B, int causal, float scale, void* Y_f16,
                           int64_t ldy, void* stream) {
  using namespace smoothrot;
  using namespace smoothrot::prefill;
  if (total_q < 0 || total_k < 0 || total_q > INT32_MAX || total_k > INT32_MAX || B < 0 || B > 65535) return SMOOTHROT_INVALID_ARG;
  if (n_heads <= 0 || n_kv_heads <= 0 || n_heads > 65535 || n_heads % n_kv_heads != 0) return SMOOTHROT_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return SMOOTHROT_UNSUPPORTED_K;
  if ((causal & ~1) != 0 || !(scale == scale)) return SMOOTHROT_INVALID_ARG;
  if (total_q == 0 || B == 0) return SMOOTHROT_OK;
  const int64_t cq = n_heads * head_dim, ckv = n_kv_heads * head_dim;
  if (Q_f16 == nullptr || Y_f16 == nullptr || cu_q == nullptr || cu_k == nullptr || ldq < cq || ldy < cq) return SMOOTHROT_INVALID_ARG;
  if (total_k > 0 && (K_f16 == nullptr || V_f16 == nullptr || ldk < ckv || ldv < ckv)) return SMOOTHROT_INVALID_ARG;
  if (!aligned16(Q_f16) || !aligned16(Y_f16) || ldq % 8 != 0 || ldy % 8 != 0) return SMOOTHROT_BAD_ALIGNMENT;
  if (total_k > 0 && (!aligned16(K_f16) || !aligned16(V_f16) || ldk % 8 != 0 || ldv % 8 != 0)) return SMOOTHROT_BAD_ALIGNMENT;
  Args a;
  a.q = static_cast<const __half*>(Q_f16); a.k = static_cast<const __half*>(K_f16); a.v = static_cast<const __half*>(V_f16);
  a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldy = ldy;
  a.y = static_cast<__half*>(Y_f16);
  a.total_q = total_q; a.total_k = total_k;
  a.cu_q = cu_q; a.cu_k = cu_k;
  a.batch = int(B); a.n_heads = int(n_heads); a.group = int(n_heads / n_kv_heads); a.causal = causal;
  a.scale = scale;
  const dim3 grid(unsigned((total_q + kWarps - 1) / kWarps), unsigned(n_heads));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (head_dim == 128) attn_prefill_kernel<128><<<grid, 32 * kWarps, 0, st>>>(a);
  else attn_prefill_kernel<64><<<grid, 32 * kWarps, 0, st>>>(a);
  count_launch();
  return launch_status();
}

}  // extern "C"
