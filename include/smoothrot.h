/*
 * libsmoothrot: the W4A4 SmoothRot linear layer on one NVIDIA B200 (sm_100a).
 *
 * The library implements the quantized linear layer that the SmoothRot method
 * produces.  Notation (the paper's, with PyTorch's weight layout):
 *
 *   X  [M x K] fp16   activations, one row per token (K = input channels)
 *   W  [N x K] fp16   weights, one row per output channel;  Y = X W^T
 *   s  [K]     fp32   smoothing scales, Lambda = diag(s)
 *   d  [K]     fp32   +1/-1 sign diagonal that randomises the Hadamard matrix
 *   H          +1/-1  Hadamard matrix of order K (H H^T = K I):
 *                     K = 2^p : Sylvester / Walsh, H[i][j] = (-1)^popcount(i & j)
 *                     K = 28 * 2^p : kron(H28, H_{2^p}), index j = a * 2^p + b,
 *                     H28 = Paley construction I over GF(27) (smoothrot_paley28)
 *                     K = 12 * 2^p, 20 * 2^p : the same with Paley I over GF(11), GF(19)
 *                     (smoothrot_base_matrix; an addition for other layer widths, the
 *                     paper's models need only the two forms above)
 *
 * The equivalent transformation (Eq. 2 of the paper) is
 *   Y = (X diag(pre_x) H / sqrt(K)) (W diag(pre_w) H / sqrt(K))^T,
 *   pre_x = d / s,  pre_w = s * d,
 * i.e. A = (H Lambda)^-1 of the Methodology section with the random signs
 * merged into the diagonal.  Both factors are quantized to signed 4-bit codes
 * (Eq. 1, symmetric form, codes in [-8, 7]) with one fp32 step size per row.
 *
 * Packed INT4 layout (used for Xq and Wq): row-major, K/2 bytes per row; byte
 * i of a row holds code 2i in bits 0-3 and code 2i+1 in bits 4-7, each as
 * 4-bit two's complement.
 *
 * Conventions for every call
 *   - All tensor pointers are DEVICE pointers unless marked "host".  The
 *     caller owns every buffer; the library allocates nothing and keeps no
 *     reference after the work it enqueued has run.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).
 *     Calls only enqueue work; they do not synchronise.
 *   - Leading dimensions (ldx, ldw, ldy) count elements, not bytes.
 *   - fp16 inputs must be 16-byte aligned with leading dimensions that are
 *     multiples of 8; packed tensors must be 16-byte aligned.
 *   - K must be 2^p with 7 <= p <= 13, or 12 * 2^p, 20 * 2^p or 28 * 2^p with 3 <= p <= 10.
 *   - Return value: SMOOTHROT_OK (0) or a negative smoothrot_status.  On an
 *     error nothing has been enqueued.  A size of zero rows is valid and
 *     enqueues nothing.
 */
#ifndef SMOOTHROT_H_
#define SMOOTHROT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SMOOTHROT_OK = 0,
  SMOOTHROT_INVALID_ARG = -1,         /* null pointer, negative size, bad ratio */
  SMOOTHROT_UNSUPPORTED_K = -2,       /* K is not one of the supported orders */
  SMOOTHROT_BAD_ALIGNMENT = -3,       /* pointer or leading dimension misaligned */
  SMOOTHROT_WORKSPACE_TOO_SMALL = -4, /* see smoothrot_workspace_bytes */
  SMOOTHROT_CUDA_ERROR = -5,          /* a CUDA runtime / driver call failed */
  SMOOTHROT_DEVICE_TIMEOUT = -6,      /* a bounded wait inside a kernel ran out */
  SMOOTHROT_STATIC_SCRATCH_EXCEEDED = -7 /* shape needs more than SMOOTHROT_STATIC_SCRATCH_BYTES */
} smoothrot_status;

/* Host. Text for a status code; never NULL. */
const char* smoothrot_status_string(int status);

/*
 * Scale calibration.  Methodology section:
 *     s_j = max|X_j|^alpha / max|W_j|^(1 - alpha)
 * with max|X_j| taken over all calibration tokens of the layer's raw input
 * and max|W_j| over the output channels of the original weights.
 *
 * Call once per calibration batch.  Every call folds the batch into the
 * running per-channel maximum  amax[j] = max(amax[j], max_t |X[t][j]|);
 * the caller zero-fills amax before the first batch.  X may be NULL with
 * T = 0.  When `finalize` is non-zero the call also reads W [N x K] and writes
 *     s[j]     = max(amax[j], eps)^alpha / max(wmax[j], eps)^(1 - alpha),
 *                floored at eps = 1e-5  (fp64 arithmetic, rounded to fp32)
 * and, if `d` is non-NULL, the two diagonals the other calls take:
 *     pre_w[j] = s[j] * d[j]          (for smoothrot_fuse_weights)
 *     pre_x[j] = d[j] / s[j]          (for smoothrot_quant_act)
 * pre_w_out / pre_x_out may each be NULL.  s_out doubles as the scratch for
 * max|W_j| while the call runs.  W, s_out are ignored when finalize == 0.
 */
int smoothrot_calibrate(const void* X_f16, int64_t T, int64_t K, int64_t ldx,
                        const void* W_f16, int64_t N, int64_t ldw,
                        float alpha, int finalize,
                        float* amax_inout, float* s_out,
                        const float* d, float* pre_w_out, float* pre_x_out,
                        void* stream);

/*
 * Offline weight path (Methodology section; Fig. 2's down-projection block
 * "H Lambda W"; Experimental settings, "Quantization": per-channel symmetric
 * round-to-nearest 4-bit weights).  For every row n of W:
 *     w^   = (W[n][:] * pre) H / sqrt(K)            pre = s * d, or NULL = ones
 *     dw[n]= clip_w * max|w^| / 7                   (1.0 if the row is all zero)
 *     code = clamp(round_half_even(w^ / dw[n]), -8, 7),  packed 2 per byte
 * Wq_out is [N x K/2] bytes, dw_out [N] fp32.  0 < clip_w <= 1.
 */
int smoothrot_fuse_weights(const void* W_f16, int64_t N, int64_t K, int64_t ldw,
                           const float* pre, float clip_w,
                           uint8_t* Wq_out, float* dw_out, void* stream);

/*
 * Offline weight path with the clip-ratio search of the paper's weight quantizer (Experimental
 * settings, "Quantization": per-channel symmetric weights; each clip ratio is the candidate with the
 * least squared quantization error, the candidates being tried one after another).  As smoothrot_fuse_weights, but for every row
 * the ratio is chosen from the grid
 *     ratio_i = fp32(1 - i * (1 - lowest_ratio) / (ratio_count - 1)),   i = 0 .. ratio_count - 1
 * (the paper gives no grid; 1.00 .. 0.50 in 51 steps is what the tests and the oracle use) as the
 * first i that minimises  sum_k (w^_k - code_k * step_i)^2,  step_i = fp32(ratio_i * max|w^|) / 7,
 * with the codes of Eq. 1's symmetric quantizer at that step; the error is summed in fp64.
 * best_out [N] int32 (may be NULL) receives the chosen i.  `workspace` holds the rotated fp32
 * rows: smoothrot_fuse_weights_search_workspace_bytes(N, K) bytes for one pass, or any multiple
 * of 4 K bytes (at least one row) to work in slices.  0 < lowest_ratio <= 1, 1 <= ratio_count <= 1024.
 */
size_t smoothrot_fuse_weights_search_workspace_bytes(int64_t N, int64_t K);
int smoothrot_fuse_weights_search(const void* W_f16, int64_t N, int64_t K, int64_t ldw,
                                  const float* pre, float lowest_ratio, int ratio_count,
                                  uint8_t* Wq_out, float* dw_out, int32_t* best_out,
                                  void* workspace, size_t workspace_bytes, void* stream);

/*
 * Online activation path (Fig. 2, "hadamard" then "quantize" before the
 * down-projection; Experimental settings, "Quantization": per-token symmetric
 * 4-bit activations with a constant clip ratio, 0.9 in the paper).  For every
 * token m:
 *     x^   = (X[m][:] * pre) H / sqrt(K)            pre = d / s, or NULL when
 *                                                   Lambda^-1 already sits in
 *                                                   the producing layer
 *     dx[m]= clip_a * max|x^| / 7                   (1.0 if the row is all zero)
 *     code = clamp(round_half_even(x^ / dx[m]), -8, 7),  packed 2 per byte
 * Xq_out is [M x K/2] bytes, dx_out [M] fp32.  0 < clip_a <= 1.
 */
int smoothrot_quant_act(const void* X_f16, int64_t M, int64_t K, int64_t ldx,
                        const float* pre, float clip_a,
                        uint8_t* Xq_out, float* dx_out, void* stream);

/*
 * Online activation quantizer of the layers that have no online Hadamard transform.  Methodology
 * section, last paragraph: every quantized layer quantizes its activations online, in the forward
 * pass, while only two layers also rotate them there (smoothrot_quant_act and
 * smoothrot_quant_act_heads); every other quantized layer receives activations that are already
 * in the rotated basis.  For every token m:
 *     x^   = X[m][:] * pre                       (pre [K] fp32, or NULL for none)
 *     dx[m], codes: from x^ exactly as in smoothrot_quant_act.
 * X [M x ldx] fp16, Xq_out [M x K/2] bytes, dx_out [M] fp32.  K a multiple of 8, K <= 16384.
 */
int smoothrot_quant_act_plain(const void* X_f16, int64_t M, int64_t K, int64_t ldx,
                              const float* pre, float clip_a,
                              uint8_t* Xq_out, float* dx_out, void* stream);

/*
 * Online activation path in front of the attention output projection.  Methodology section: the
 * forward pass contains two online Hadamard transforms, for which the paper defers to QuaRot; it
 * spells out only the one before the down-projection (smoothrot_quant_act).  The other
 * one, as QuaRot describes it, mixes the heads of the attention output: a row of X is the
 * concatenation of n_heads head outputs of head_dim values, and
 *     x^[m][g * head_dim + e] = sum_h X[m][h * head_dim + e] * pre[h * head_dim + e] * H[h][g] / sqrt(n_heads)
 * with H the Sylvester matrix of order n_heads, i.e. the row times (H_heads (x) I_head_dim) /
 * sqrt(n_heads); the per-head factor (I (x) H_head_dim) of the full rotation is folded into the
 * value projection offline.  The transform is exact in the paper's setting, so `pre` is normally
 * NULL.  dx and the codes follow from x^ exactly as in smoothrot_quant_act.
 * X is [M x ldx] fp16 with ldx >= K = n_heads * head_dim, Xq_out [M x K/2] bytes, dx_out [M] fp32.
 * Supported: n_heads in {8, 16, 32, 64}, head_dim in {64, 128, 256} (else SMOOTHROT_UNSUPPORTED_K).
 */
int smoothrot_quant_act_heads(const void* X_f16, int64_t M, int64_t n_heads, int64_t head_dim, int64_t ldx,
                              const float* pre, float clip_a,
                              uint8_t* Xq_out, float* dx_out, void* stream);

/*
 * The online activation path fed directly by the gated linear unit (Fig. 2: the edge
 * "sigma(gate) (.) up -> hadamard -> quantize" in front of the down-projection; Methodology
 * section: Lambda^-1 is absorbed into the up-projection because the gated product is
 * channel-wise, so `pre` is normally NULL or the sign diagonal alone).  Same as
 * smoothrot_quant_act on X[m][j] = SiLU(gate[m][j]) * up[m][j], SiLU(g) = g / (1 + exp(-g)),
 * except that X is formed in fp32 inside the kernel and never rounded to fp16 or written to
 * memory.  gate, up: [M x K] fp16 with leading dimensions ld_gate, ld_up (multiples of 8,
 * 16-byte aligned rows).  K = 14336 runs the dedicated kernel; other supported K run the generic
 * one-row-per-block kernel.
 */
int smoothrot_quant_act_glu(const void* gate_f16, const void* up_f16, int64_t M, int64_t K,
                            int64_t ld_gate, int64_t ld_up, const float* pre, float clip_a,
                            uint8_t* Xq_out, float* dx_out, void* stream);

/*
 * The quantized layer (Eq. 2's product on the integer codes of Eq. 1, then
 * Eq. 1's dequantizer Q(x) = x_int * step applied to both factors):
 *     acc[m][n] = sum_k Xq[m][k] * Wq[n][k]                    (int32, exact)
 *     Y[m][n]   = fp16( float(acc[m][n]) * dx[m] * dw[n] )
 * Xq [M x K/2], Wq [N x K/2] packed; dx [M], dw [N] fp32; Y [M x ldy] fp16
 * with ldy >= N, ldy a multiple of 8, Y 16-byte aligned.  K must be a multiple
 * of 128 and at most 65536; any M >= 0 and any N >= 0 that is a multiple of 8.
 * `workspace` must hold smoothrot_workspace_bytes(M, N, K) bytes (it may be
 * NULL when that is 0); its contents on entry do not matter.
 */
int smoothrot_linear(const uint8_t* Xq, const float* dx, int64_t M,
                     const uint8_t* Wq, const float* dw, int64_t N, int64_t K,
                     void* Y_f16, int64_t ldy,
                     void* workspace, size_t workspace_bytes, void* stream);

/*
 * smoothrot_linear without a caller-provided workspace.  (An addition of this
 * library; the paper has no counterpart.)
 *
 * Who needs it: code that must run the layer but is not in a position to
 * obtain device memory for the split-K scratch.  Typical cases are a plug-in
 * inside a serving process whose host application handed out all device
 * memory at start-up and forbids cudaMalloc afterwards, a component that is
 * only ever given the input and output buffers of the layer, or a process in
 * which cudaMalloc would fail because another allocator has already reserved
 * the whole device.  For such callers the scratch lives inside the library: a
 * fixed array of SMOOTHROT_STATIC_SCRATCH_BYTES in device memory that belongs
 * to the loaded module.  Every GPU on which the library is used keeps that
 * many bytes occupied until the process exits, whether or not this entry
 * point is ever called there.
 *
 * Same arguments, results and error behaviour as smoothrot_linear (the same
 * checks in the same order, before anything else), minus the workspace pair.  The call itself allocates and frees nothing.  Shapes whose
 * smoothrot_workspace_bytes(M, N, K) exceeds SMOOTHROT_STATIC_SCRATCH_BYTES
 * are refused with SMOOTHROT_STATIC_SCRATCH_EXCEEDED and nothing is enqueued
 * (use smoothrot_linear with your own workspace for those).
 *
 * The first call on each device looks up the array's device address
 * (cudaGetSymbolAddress, with that device current) and remembers it; make that
 * first call before starting any stream capture on the device.
 *
 * There is ONE array per device, shared by every call: two calls whose work
 * may overlap on the GPU (different streams, or several host threads) race on
 * it and produce garbage.  Calls on one stream are safe.  The array keeps
 * whatever the previous call left; this entry point never depends on those
 * contents, because each call overwrites every partial sum it later reads.
 */
#define SMOOTHROT_STATIC_SCRATCH_BYTES (8u * 1024u * 1024u)
int smoothrot_linear_static_scratch(const uint8_t* Xq, const float* dx, int64_t M,
                                    const uint8_t* Wq, const float* dw, int64_t N, int64_t K,
                                    void* Y_f16, int64_t ldy, void* stream);

/*
 * KV-cache quantizer (Eq. 1, asymmetric form; Experimental settings, "Quantization": KV caches
 * are quantized asymmetrically with a group size of 128 and a clip ratio of 0.95).  For every
 * group of 128 consecutive values of a row of X [rows x C] fp16 (C a multiple of 128):
 *     hi = fp32(clip * max), lo = fp32(clip * min)        (the ratio shrinks both ends)
 *     step = (hi - lo) / 15                               (1.0 for a constant group)
 *     zero = -round_half_even(lo / step)
 *     code = clamp(round_half_even(x / step) + zero, 0, 15)
 * all in fp32.  q_out [rows x C/2] bytes holds the unsigned codes, value 2i in bits 0-3 and value
 * 2i+1 in bits 4-7; step_out, zero_out [rows x C/128] fp32 (zero is integer valued and may lie
 * outside 0..15 when a group does not straddle zero).  0 < clip <= 1.
 * smoothrot_kv_dequant is Eq. 1's dequantizer  Y = fp16((code - zero) * step),  Y [rows x ldy].
 */
int smoothrot_kv_quant(const void* X_f16, int64_t rows, int64_t C, int64_t ldx, float clip,
                       uint8_t* q_out, float* step_out, float* zero_out, void* stream);
int smoothrot_kv_dequant(const uint8_t* q, const float* step, const float* zero, int64_t rows,
                         int64_t C, void* Y_f16, int64_t ldy, void* stream);

/*
 * Paged key-value cache and the attention over it: the part of a decoder layer between the fused
 * QKV projection and the head-mixing quantizer in front of the output projection
 * (smoothrot_quant_act_heads), with 4-bit keys and values as in the paper's W4A4KV4 setting or fp16 ones.
 * (The paper fixes the quantizer of the cache; pages, position rotation and attention are the
 * models' own, LLaMA's and Mistral's, in their usual formulas.)
 *
 * Cache.  `bits` 16: k_cache and v_cache are fp16 [pages][n_kv_heads][page_size][head_dim].
 * `bits` 4: bytes [pages][n_kv_heads][page_size][head_dim / 2], unsigned codes, value 2i in bits 0-3 and
 * 2i+1 in bits 4-7 as in smoothrot_kv_quant, and k_params, v_params fp32
 * [pages][groups][page_size][2] hold the step and the zero point of each group of 128 values of a
 * token's row of n_kv_heads * head_dim values (groups = n_kv_heads * head_dim / 128; with heads of
 * 64 two heads share a group, so n_kv_heads must be even).  A value is (code - zero) * step.  k_params and v_params are
 * ignored with `bits` 16.  All 16-byte aligned.  page_size is a power of two up to 1024, head_dim is
 * 64 or 128 (else SMOOTHROT_UNSUPPORTED_K); n_kv_heads * page_size * head_dim * 2 must stay below 2^31.
 * A slot is page * page_size + offset; offsets into a cache are 64-bit.
 *
 * Values that only the device sees (slots, positions, pages, lengths) are checked by the kernels: what is out of range is
 * left out as each call says, nothing is read or written outside the buffers, and smoothrot_device_status reports
 * a code: 32 to 35, named at each call, or 36 to 41 when a bounded wait inside an attention kernel has run out (its
 * output is then incomplete).
 */

/*
 * Appends T tokens.  Row t of Q [T x ldq], K [T x ldk], V [T x ldv] (fp16, e.g. the three slices of the
 * fused projection's output row) holds the token's n_heads query heads, n_kv_heads key heads and
 * value heads.  Queries and keys are rotated by the token's position p = positions[t]:
 *     a' = a cos(p, i) - b sin(p, i),  b' = b cos(p, i) + a sin(p, i)          (fp32, each product rounded)
 * for the pairs (a, b) = (x[i], x[i + head_dim/2]), or (x[2i], x[2i+1]) with `interleaved` = 1;
 * rotary [rotary_rows x head_dim] fp32 holds head_dim/2 cosines and then head_dim/2 sines per position.
 * With `walsh` = 1 every query and key head is then multiplied by H_head_dim / sqrt(head_dim) (Walsh): products of
 * queries and keys stay what they are, and key outliers are spread before they are coded.
 * The results: Q_out [T x ldqo] fp16; K_out [T x ldko] fp16 if not NULL; keys and values at slots[t] of the
 * cache, 4-bit codes with smoothrot_kv_quant's formulas (the keys' from the fp32 values after the rotation) at
 * clip ratio `clip`.  A negative slot: rotated, not cached.  A token whose position is outside
 * [0, rotary_rows) or whose slot is beyond the cache: nothing of it is written, status code 32.
 * Two tokens of one call must not share a slot.  n_heads may be 0 (keys and values alone; Q, Q_out ignored).
 * Q_out may be Q and K_out may be K (same leading dimension).
 */
int smoothrot_kv_append(const void* Q_f16, int64_t ldq, const void* K_f16, int64_t ldk,
                        const void* V_f16, int64_t ldv, int64_t T, int64_t n_heads,
                        int64_t n_kv_heads, int64_t head_dim, const int32_t* positions,
                        const float* rotary, int64_t rotary_rows, int interleaved, int walsh,
                        void* Q_out_f16, int64_t ldqo, void* K_out_f16, int64_t ldko,
                        const int64_t* slots, int bits, int64_t pages, int64_t page_size,
                        void* k_cache, void* v_cache, float* k_params, float* v_params,
                        float clip, void* stream);

/*
 * Reads T rows of the cache back: K_out [T x ldk], V_out [T x ldv] fp16, row t from slots[t], 4-bit
 * codes as smoothrot_kv_dequant turns them into values.  For a later chunk of a prompt, whose
 * queries attend to the cached prefix through smoothrot_attn_prefill.  A negative slot gives a row of zeros, one
 * beyond the cache zeros and status code 33.  T * n_kv_heads * head_dim / 128 must stay below 2^31.
 */
int smoothrot_kv_gather(const int64_t* slots, int64_t T, int64_t n_kv_heads, int64_t head_dim,
                        int bits, int64_t pages, int64_t page_size, const void* k_cache,
                        const void* v_cache, const float* k_params, const float* v_params,
                        void* K_out_f16, int64_t ldk, void* V_out_f16, int64_t ldv, void* stream);

/*
 * Attention of one new token of each of B sequences over the cache.  For sequence b and query head h,
 * over the tokens j < lengths[b] of key head h / (n_heads / n_kv_heads):
 *     y = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale * q.k_j - max)
 * with fp32 scores, statistics and sums; y = 0 for an empty sequence.  Token j of sequence b lies in page
 * block_table[b * max_pages + j / page_size] at offset j % page_size.  Q [B x ldq] and Y [B x ldy] fp16
 * rows of n_heads * head_dim values; n_heads a multiple of n_kv_heads; B <= 8192, max_pages * page_size < 2^31 and
 * B * (max_pages * page_size / 16 + 2) * n_kv_heads * ceil(n_heads / n_kv_heads / 16) < 2^31.
 * A length outside [0, max_pages * page_size] is clamped and a token on a page outside [0, pages) left out, both
 * with status code 34; y = 0 where none is left.  Weights are rounded to fp16 before they multiply the values: 11 bits down to
 * 2^-21 of the largest, counted down to 2^-31; with `bits` 4 of the weight times the value's step, so tokens whose steps
 * are more than 2^21 below another's lose bits.  The order of all sums is fixed by the shapes and lengths: a call repeated gives the same bits.
 * `workspace`: smoothrot_attn_decode_workspace_bytes(...) bytes, 16-byte aligned, contents on entry do not matter; calls
 * that may overlap on the GPU need one each.
 */
size_t smoothrot_attn_decode_workspace_bytes(int64_t B, int64_t n_heads, int64_t n_kv_heads,
                                             int64_t head_dim);
int smoothrot_attn_decode(const void* Q_f16, int64_t ldq, int64_t B, int64_t n_heads,
                          int64_t n_kv_heads, int64_t head_dim, int bits, int64_t pages,
                          int64_t page_size, const void* k_cache, const void* v_cache,
                          const float* k_params, const float* v_params,
                          const int32_t* block_table, int64_t max_pages, const int32_t* lengths,
                          float scale, void* Y_f16, int64_t ldy, void* workspace,
                          size_t workspace_bytes, void* stream);

/*
 * Attention over B packed sequences: sequence b has the queries cu_q[b] .. cu_q[b+1]-1 and the keys and values
 * cu_k[b] .. cu_k[b+1]-1 (int32, device, B + 1 entries, not decreasing).  The same formula as above over the
 * keys of the query's sequence, with `causal` = 1 over those with j <= i + keys - queries (i, j from the
 * sequence's start): the sequences' ends are aligned, a prefix of earlier keys is visible to all, and a
 * query that sees no key gives y = 0.  What a query does not see has no part in its output, whatever its values.
 * Q [total_q x ldq], K [total_k x ldk], V [total_k x ldv], Y [total_q x ldy] fp16 rows of heads.
 * Weights are rounded to fp16 as above (`bits` 16).
 * Rows that belong to no sequence are not written; a sequence that leaves the buffers is left out, status code 35.
 * total_q, total_k <= 2^30, B <= 65535.
 */
int smoothrot_attn_prefill(const void* Q_f16, int64_t ldq, int64_t total_q, const void* K_f16,
                           int64_t ldk, const void* V_f16, int64_t ldv, int64_t total_k,
                           int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                           const int32_t* cu_q, const int32_t* cu_k, int64_t B, int causal,
                           float scale, void* Y_f16, int64_t ldy, void* stream);

/*
 * Microscaled 4-bit floating point: the same layers with codes that the tensor cores multiply as they are.  (An addition of
 * this library; the paper's codes are integers with a step per row.)
 *
 * A code is e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign in bit 3, two to a byte along the row, value 2i in bits 0-3.
 * Conversions round to the nearest, ties to the even code, and saturate at 6.  A value is code * scale (* step):
 *   group 32: a scale per 32 neighbouring values, a power of two, held as exponent + 127 in a byte (255: NaN);
 *             steps are not needed
 *   group 16: a scale per 16 neighbouring values, e4m3, and a step per row, fp32
 * Codes are [rows x K/2] bytes.  Scales lie in blocks of 512 bytes for 128 rows and 4 neighbouring groups, blocks along
 * the row first: row r and group g are at
 *     ((r / 128) * (K / group / 4) + g / 4) * 512 + (r % 32) * 16 + (r % 128) / 32 * 4 + g % 4
 * of smoothrot_mx_scale_bytes(rows, K, group) bytes.  Bytes of rows past the last are not written, and their contents do
 * not matter to the calls that read the rest.  Codes, scales and fp32 vectors along channels (pre, steps of weights, weights
 * of norms) are 16-byte aligned, K is a multiple of 128.
 */

/* Host. Bytes of the scales of `rows` rows of K values; 0 for a group or K that is not supported. */
size_t smoothrot_mx_scale_bytes(int64_t rows, int64_t K, int64_t group);

/*
 * Quantizer, for weights and activations alike.  For every row, in fp32, each product and sum rounded by itself:
 *     v = X[m][:] * pre                                    pre [K] or NULL: d / s or s * d as in smoothrot_quant_act
 *     v = v (I (x) H_n) / sqrt(n)                          n = walsh: Walsh rotation of blocks of 32, 64 or 128, 0: none
 *     group 32: scale = 2^E with the least E such that max|v of the group| <= 7 * 2^E, -127 <= E  (2^0 for a group of zeros)
 *               code = e2m1(v / scale)
 *     group 16: step[m] = the least power of two with max|v of the row| <= 2688 * step, at least 2^-100  (1 for zeros)
 *               scale = e4m3(max|v of the group| / (6 step)),  code = e2m1(v / (scale * step)), 0 where the scale is 0
 * X rotated in blocks of n needs weights that are rotated in the same blocks.  An infinity or NaN makes its group's
 * scale (group 32) or its row's step (group 16) NaN, and with it every product that it takes part in.
 * X [M x ldx] fp16; step_out [M] with group 16, NULL with 32.  K <= 32768.
 */
int smoothrot_mx_quant(const void* X_f16, int64_t M, int64_t K, int64_t ldx, int64_t group, const float* pre, int walsh,
                       uint8_t* q_out, uint8_t* scale_out, float* step_out, void* stream);

/* Codes back to values: Y[m][k] = fp16(code * (scale * step[m])), step NULL: 1.  Y [M x ldy] fp16. */
int smoothrot_mx_dequant(const uint8_t* q, const uint8_t* scale, const float* step, int64_t M, int64_t K, int64_t group,
                         void* Y_f16, int64_t ldy, void* stream);

/*
 * The layer on microscaled codes:
 *     Y[m][n] = fp16( (sum over groups of x_scale w_scale (sum of x w)) * (x_step[m] * w_step[n]) )     fp32 sums
 * Xq, x_scale [M rows], Wq, w_scale [N rows], both of K values in groups of `group`; x_step [M], w_step [N] or NULL (1).
 * Y [M x ldy] fp16.  Any M >= 0, N a multiple of 8, K <= 2^20.  A call repeated gives the same bits.  No workspace.
 */
int smoothrot_mx_linear(const uint8_t* Xq, const uint8_t* x_scale, const float* x_step, int64_t M, const uint8_t* Wq,
                        const uint8_t* w_scale, const float* w_step, int64_t N, int64_t K, int64_t group, void* Y_f16,
                        int64_t ldy, void* stream);

/*
 * Both projections of a gated feed-forward block, its activation and product in one kernel:
 *     h[m][f] = SiLU(gate) * up,  gate = x . gate_row[f],  up = x . up_row[f]  as in smoothrot_mx_linear, in fp32
 *     walsh = 32: h rotated in blocks of 32 neighbouring features by H_32 / sqrt(32), for a down projection whose
 *                 weights went through smoothrot_mx_quant with walsh = 32;  0: none
 * and either H [M x ldh] = fp16(h), or, with q_out and scale_out in place of H, h in codes for the down projection, as
 * smoothrot_mx_quant makes them except that with group 16 the steps h_step [M] are the caller's (calibrated: a row's
 * maximum is not known while its first features leave), from 2^-100 to 2^117 as the quantizer's own are; where a row's values
 * exceed 2688 steps they saturate with their sign, but an infinity or NaN makes its group's scale NaN.  h_step is NULL with group 32.  F a multiple of 8, of 32 with walsh, of 128 with codes.
 * A diagonal on h, in front of the rotation, goes into up_step.
 */
int smoothrot_mx_glu(const uint8_t* Xq, const uint8_t* x_scale, const float* x_step, int64_t M, const uint8_t* gate_q,
                     const uint8_t* gate_scale, const float* gate_step, const uint8_t* up_q, const uint8_t* up_scale,
                     const float* up_step, int64_t F, int64_t K, int64_t group, int walsh, void* H_f16, int64_t ldh,
                     uint8_t* q_out, uint8_t* scale_out, const float* h_step, void* stream);

/*
 * The residual stream between two blocks, with the norms after the one and before the other:
 *     z = Y[m][:],  with post_norm = 1:  z = Y * rstd(Y) * post_w                     post_w [K] or NULL: 1
 *     H' = fp16( residual_scale * H + block_scale * (gate * z) )                      gate [K] or NULL: 1
 *     x = fp16( H' * rstd(H') * pre_w )                                               pre_w [K] or NULL: 1
 *     rstd(r) = 1 / sqrt(mean(r^2) + eps), the mean in more than 32 bits, rstd rounded to fp32;
 *     products from the left, each and the sum rounded to fp32 by itself
 * Y NULL: H' = fp16(residual_scale * H), H NULL: H' = fp16(block_scale * (gate * z)).  Written are, of H_out [M x ldho], X_out [M x ldxo]
 * (fp16) and the codes of x, those that are asked for: `codes` 0 none; 4 what smoothrot_quant_act_plain makes of X_out
 * with ratio `clip` (step_out: dx_out), except that a NaN in a row makes its step NaN; 16 or 32 what smoothrot_mx_quant makes of
 * X_out in groups of that size.
 * H_out may be H or Y and X_out may be H or Y, with the same leading dimension, but not one and the same.  q_out and step_out go with
 * codes, scale_out with codes 16 and 32; where they are not asked for they are NULL.
 * K a multiple of 8, of 128 with codes 16 and 32; K <= 32768.  eps > 0.
 */
int smoothrot_add_norm(const void* Y_f16, int64_t ldy, const void* H_f16, int64_t ldh, int64_t M, int64_t K, int post_norm,
                       const float* post_w, const float* gate, float block_scale, float residual_scale,
                       const float* pre_w, float eps, void* H_out_f16, int64_t ldho, void* X_out_f16, int64_t ldxo,
                       int codes, float clip, uint8_t* q_out, uint8_t* scale_out, float* step_out, void* stream);

/*
 * The whole online layer for a handful of tokens in one kernel: the online activation path
 * followed by smoothrot_linear (Fig. 2: ["hadamard" ->] "quantize" -> the quantized projection; Eq. 2
 * on Eq. 1's integer codes), for decode steps, where two launches cost more than the work.  Every
 * CTA prepares the tokens for itself while its share of the weights is in flight.
 *   rotation = 1: the tokens go through smoothrot_quant_act's path (x * pre) H / sqrt(K), same
 *                 formulas, fp32 butterflies in a different order of additions.  K = 4096, M <= 4.
 *   rotation = 0: through smoothrot_quant_act_plain's path (x * pre, no rotation), same codes.
 *                 K in {1024, 2048, 4096}, M <= 8.
 * The codes and steps are written to Xq_out [M x K/2] / dx_out [M] when those are non-NULL (device,
 * optional).  X [M x ldx] fp16, pre [K] or NULL, Wq [N x K/2] and dw [N] from
 * smoothrot_fuse_weights, Y [M x ldy] fp16, N a multiple of 8.  Other shapes:
 * SMOOTHROT_INVALID_ARG (M) / SMOOTHROT_UNSUPPORTED_K.  No workspace.
 */
int smoothrot_linear_decode(const void* X_f16, int64_t M, int64_t K, int64_t ldx, int rotation,
                            const float* pre, float clip_a, const uint8_t* Wq, const float* dw,
                            int64_t N, void* Y_f16, int64_t ldy, uint8_t* Xq_out, float* dx_out,
                            void* stream);

/* As smoothrot_linear_decode, for the attention output projection: the tokens go through
 * smoothrot_quant_act_heads' path, (x * pre)(H_heads (x) I_head_dim) / sqrt(heads).  Supported:
 * 32 heads of 128 (K = 4096), M <= 4. */
int smoothrot_linear_decode_heads(const void* X_f16, int64_t M, int64_t n_heads, int64_t head_dim,
                                  int64_t ldx, const float* pre, float clip_a, const uint8_t* Wq,
                                  const float* dw, int64_t N, void* Y_f16, int64_t ldy,
                                  uint8_t* Xq_out, float* dx_out, void* stream);

/* Host. Scratch bytes smoothrot_linear / smoothrot_debug_gemm_i32 want for
 * this shape (0 for shapes that need none).  With M <= 128 a shape that reports
 * a size cannot run without it (SMOOTHROT_WORKSPACE_TOO_SMALL).  With M >= 256 the
 * scratch only serves to split K over otherwise idle SMs (few output tiles, long
 * K): with a smaller or absent workspace the call runs unsplit, slower but with
 * the same result. */
size_t smoothrot_workspace_bytes(int64_t M, int64_t N, int64_t K);

/* Host. Name of the kernel (or kernel pair) smoothrot_linear launches for this shape when it is
 * given the workspace smoothrot_workspace_bytes reports: a static string, "none" for shapes the
 * call rejects.  For reports and benchmarks; nothing is launched. */
const char* smoothrot_linear_plan_name(int64_t M, int64_t N, int64_t K);

/*
 * Test exports: values the fused kernels never write to memory.
 *   smoothrot_debug_hadamard: Y[m][:] = (X[m][:] * pre) H / sqrt(K) as fp32
 *     [M x K], the rotation alone (Methodology section).
 *   smoothrot_debug_hadamard_heads: the same for the head-mixing transform of
 *     smoothrot_quant_act_heads, Y [M x n_heads * head_dim] fp32.
 *   smoothrot_debug_gemm_i32: the int32 accumulators acc [M x N] of
 *     smoothrot_linear, computed by the same kernels.
 */
int smoothrot_debug_hadamard(const void* X_f16, int64_t M, int64_t K, int64_t ldx,
                             const float* pre, float* Y_f32, void* stream);
int smoothrot_debug_hadamard_heads(const void* X_f16, int64_t M, int64_t n_heads, int64_t head_dim,
                                   int64_t ldx, const float* pre, float* Y_f32, void* stream);
int smoothrot_debug_gemm_i32(const uint8_t* Xq, int64_t M, const uint8_t* Wq, int64_t N,
                             int64_t K, int32_t* acc,
                             void* workspace, size_t workspace_bytes, void* stream);

/*
 * Test exports for the bounded device-side waits (no passage of the paper: the kernels never
 * spin without bound, and these two calls let a test see a wait run out without hanging
 * anything).
 *   smoothrot_debug_set_wait_limit_ns: host, synchronous.  Sets the limit of every bounded wait
 *     of the library's kernels on the current device, in nanoseconds; 0 restores the default
 *     (two seconds).  Below 1000 the attention kernels take their first wait as run out at once: their output
 *     is then missing, and smoothrot_device_status reports 36 or 41.
 *   smoothrot_debug_wait_expiry: enqueues one warp that waits, through the same bounded wait as
 *     the GEMM kernels, on a barrier nobody arrives on.  When the limit has passed the warp
 *     records code 7 in the status word smoothrot_device_status reads, and the kernel returns.
 *   smoothrot_debug_attn_wait_expiry: the same through the waits of the attention kernels; `code` is the one to record,
 *     36 to 40 for smoothrot_attn_prefill's and 41 for smoothrot_attn_decode's.
 *   smoothrot_debug_mx_wait_expiry: the same through the waits of the microscaled products, code 50.
 *   smoothrot_debug_norm_wait_expiry: the same through smoothrot_add_norm's wait for rows, code 51.
 */
int smoothrot_debug_set_wait_limit_ns(uint64_t ns);
int smoothrot_debug_wait_expiry(void* stream);
int smoothrot_debug_attn_wait_expiry(int code, void* stream);
int smoothrot_debug_mx_wait_expiry(void* stream);
int smoothrot_debug_norm_wait_expiry(void* stream);

/* Host. Writes the library's own order-28 Paley matrix, row-major, entries
 * +1 / -1, into out[784] (a host buffer). */
int smoothrot_paley28(int8_t* out_host);

/* Host. The same for the small factor of order 12, 20 or 28 (Paley construction I over GF(11),
 * GF(19), GF(27); first row all +1, first column +1 then -1): order * order entries, row-major,
 * into a host buffer.  SMOOTHROT_INVALID_ARG for another order or a null pointer. */
int smoothrot_base_matrix(int order, int8_t* out_host);

/*
 * Host, synchronous.  Kernels never spin without bound: a wait that runs out
 * records a non-zero code in a device-side status word and the kernel
 * returns (42 to 49 in the microscaled products, 51 in smoothrot_add_norm); the cache and attention calls record 32 to 35 for a slot, position, page or
 * length out of range.  This call copies that word for the current device into
 * *status_host (0 = none so far) and clears it when `clear` is non-zero.
 */
int smoothrot_device_status(int* status_host, int clear);

/* Host. Number of kernels this library has launched since it was loaded
 * (all devices, all streams); used by the benchmark's launch count. */
int64_t smoothrot_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* SMOOTHROT_H_ */
