// What the paged key-value cache's kernels share: the cache's layout, the checks of its description, and the
// status word for what only the device can see (a slot, a page or a length out of range).
//
// Layout: [page][kv head][offset in the page][value], one tensor for keys and one for values.  A
// page of one head is contiguous, so that the attention over one head streams runs of
// page_size * head_dim values.  With 4-bit codes a row of a head is head_dim / 2 bytes, and the step and zero
// point of each group of 128 values of a token's row (one head of 128, or two heads of 64) lie as
// a pair of floats at [page][group][offset][2].
#pragma once

#include "common.cuh"

namespace smoothrot {
namespace paged {

constexpr int kGroup = 128;

struct Cache {
  void* k;
  void* v;
  float2* k_params;   // (step, zero) pairs; null with fp16 values
  float2* v_params;
  int64_t pages;
  int page_size;      // a power of two
  int page_shift;
  int kv_heads;
  int groups;         // kv_heads * head_dim / 128, 4-bit caches only
  int head_dim;
};

enum Code { kAppendRange = 32, kGatherRange = 33, kDecodeRange = 34, kPrefillRange = 35 };

// Index of the row (page, head, offset) in units of one head's row.
__device__ __forceinline__ int64_t head_row(const Cache& c, int64_t page, int head, int offset) {
  return ((page * c.kv_heads + head) << c.page_shift) + offset;
}
__device__ __forceinline__ int64_t param_row(const Cache& c, int64_t page, int group, int offset) {
  return ((page * c.groups + group) << c.page_shift) + offset;
}

// Checks of the arguments that describe a cache, in the library's order: sizes, widths, then (through
// check_pointers, which callers reach only if there is work) null pointers and alignment.
inline int check_sizes(int64_t kv_heads, int64_t head_dim, int bits, int64_t pages, int64_t page_size) {
  if (kv_heads <= 0 || kv_heads > 65535 || pages < 0 || pages > INT32_MAX) return SMOOTHROT_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return SMOOTHROT_UNSUPPORTED_K;
  if (bits != 4 && bits != 16) return SMOOTHROT_INVALID_ARG;
  if (bits == 4 && kv_heads * head_dim % kGroup != 0) return SMOOTHROT_UNSUPPORTED_K;
  if (!is_pow2(page_size) || page_size > 1024) return SMOOTHROT_INVALID_ARG;
  if (kv_heads * page_size * head_dim * 2 > INT32_MAX) return SMOOTHROT_INVALID_ARG;   // a page's bytes
  return SMOOTHROT_OK;
}
inline int check_pointers(int bits, const void* k, const void* v, const float* k_params, const float* v_params) {
  if (k == nullptr || v == nullptr) return SMOOTHROT_INVALID_ARG;
  if (bits == 4 && (k_params == nullptr || v_params == nullptr)) return SMOOTHROT_INVALID_ARG;
  if (!aligned16(k) || !aligned16(v)) return SMOOTHROT_BAD_ALIGNMENT;
  if (bits == 4 && (!aligned16(k_params) || !aligned16(v_params))) return SMOOTHROT_BAD_ALIGNMENT;
  return SMOOTHROT_OK;
}
inline Cache make_cache(int64_t kv_heads, int64_t head_dim, int bits, int64_t pages, int64_t page_size, const void* k,
                        const void* v, const float* k_params, const float* v_params) {
  Cache c;
  c.k = const_cast<void*>(k);
  c.v = const_cast<void*>(v);
  c.k_params = reinterpret_cast<float2*>(const_cast<float*>(k_params));
  c.v_params = reinterpret_cast<float2*>(const_cast<float*>(v_params));
  c.pages = pages;
  c.page_size = int(page_size);
  c.page_shift = ilog2(page_size);
  c.kv_heads = int(kv_heads);
  c.groups = bits == 4 ? int(kv_heads * head_dim / kGroup) : 0;
  c.head_dim = int(head_dim);
  return c;
}

// The status word of one source file: reads it and, where asked, clears it.
inline int read_status_word(const int& symbol, int* out, int clear) {
  if (cudaMemcpyFromSymbol(out, symbol, sizeof(int)) != cudaSuccess) return SMOOTHROT_CUDA_ERROR;
  if (clear && *out != 0) {
    const int zero = 0;
    if (cudaMemcpyToSymbol(symbol, &zero, sizeof(int)) != cudaSuccess) return SMOOTHROT_CUDA_ERROR;
  }
  return SMOOTHROT_OK;
}

}  // namespace paged
}  // namespace smoothrot
