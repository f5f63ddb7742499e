/*
 * sp_ops.h -- operators of an encoder layer that stand by themselves: products in 8-bit integers, rotary positions, and
 * attention with capped scores, distance biases and masks.
 *
 * What a student quantised in integers (sp.h, SP_DTYPE_INT8) and one that knows positions by distance
 * (sp_set_attention_form) run inside sp_forward, for callers with tensors of their own.  Conventions are those of sp.h: 0
 * or a negative SP_E* code comes back, memory is the caller's, nothing is allocated and nothing waited for, kernels
 * are enqueued on hip_stream of the current device, and calls can be captured in graphs.  Contents of device
 * arrays are not inspected on the host; offsets that are inconsistent are clamped on the device so that no access
 * leaves the buffers described.  dtype is SP_DTYPE_FP32 or SP_DTYPE_BF16.  Strides are in elements.  None has a backward pass.
 */
#ifndef SP_OPS_H_
#define SP_OPS_H_

#include <stddef.h>
#include <stdint.h>

#include "sp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- 8-bit integers -------------------------------------------------------------------------------------------
 * A row x (a token's features, or an output channel's weights) becomes codes c and a scale s, x ~ c s.  With a = max |x|, all in
 * fp32, each operation rounded to nearest even once:
 *     s = a / 127,   r = 127 / a,   c = rint(x * r)            (so |c| <= 127)
 * a < 2^-100: s = 0 and every code 0.  A row with an infinity or a NaN: s = NaN and every code 0.
 *
 * sp_quantize_int8: rows x [rows][width] (row stride x_row, at least width) -> codes [rows][width] (row stride
 * c_row, at least width) and scales [rows].  Codes behind `width` are left as they were.
 * Errors: SP_EINVAL, SP_ESHAPE (also: rows beyond 2^26 - 4, width beyond 2^31 - 2049), SP_EHIP. */
int sp_quantize_int8(const void* x, int64_t x_row, int32_t dtype, int32_t rows, int32_t width, int8_t* codes,
                     int64_t c_row, float* scales, void* hip_stream);

/* out[t][n] = epilogue(s[t] w_scales[n] sum_k c[t][k] w_codes[n][k] + bias[n]), c and s as above from the rows of x, the sum in
 * integers (exact), the rest in fp32 (s[t] w_scales[n] first: it has to stay inside that type), rounded once to dtype.
 *   x         [tokens][width_in], row stride x_row           out  [tokens][width_out], row stride out_row; not x
 *   w_codes   [width_out][width_in], row stride w_row: a multiple of 16, 16-byte aligned, every row readable up to the next
 *             multiple of 16 of width_in (what stands there does not count); -128 is not a code
 *   bias      [width_out] or null
 *   epilogue  SP_LINEAR_PLAIN, SP_LINEAR_GELU (erf form) or SP_LINEAR_RESIDUAL (+ residual [tokens][width_out] of dtype, row
 *             stride residual_row; out may be residual with the same stride)
 *   workspace 256-byte aligned, >= sp_linear_int8_workspace_bytes(tokens, width_in)
 * tokens may be 0 (nothing is done); width_in is 1..131072, width_out at least 1.  A row with an infinity or a NaN gives a row of
 * NaN.  GELU is within 4e-7 of the erf form.  Errors: SP_EINVAL, SP_ESHAPE (also: tokens beyond 2^26 - 4, w_row beyond 2^20), SP_ENOMEM, SP_EHIP. */
enum { SP_LINEAR_PLAIN = 0, SP_LINEAR_GELU = 1, SP_LINEAR_RESIDUAL = 2 };
size_t sp_linear_int8_workspace_bytes(int32_t tokens, int32_t width_in);
int sp_linear_int8(const void* x, int64_t x_row, int32_t dtype, int32_t tokens, int32_t width_in, const int8_t* w_codes,
                   int64_t w_row, const float* w_scales, int32_t width_out, const float* bias, int32_t epilogue,
                   const void* residual, int64_t residual_row, void* out, int64_t out_row, void* workspace,
                   size_t workspace_bytes, void* hip_stream);

/* ---- rotary positions ------------------------------------------------------------------------------------------
 * Angular frequencies, radians per position, of the dim / 2 pairs of a head, and the factor on the rotated values (1 but for
 * SP_ROTARY_PARTS).  Host arrays; f_i = base^(-2 i / dim), then by scaling, for contexts `factor` (>= 1) times as long as in training:
 *   SP_ROTARY_UNSCALED  f_i
 *   SP_ROTARY_LINEAR    f_i / factor
 *   SP_ROTARY_NTK       f_i of base * factor^(dim / (dim - 2))                            (dim >= 4)
 *   SP_ROTARY_PARTS     f_i g_i + f_i / factor (1 - g_i), g_i = (trained f_i / 2 pi - 1) / 31 clipped to 0..1: pairs that turned at
 *                       most once within the `trained` positions are stretched, those of 32 turns and more are not;
 *                       the factor on the values is 1 + ln(factor) / 10
 * Errors: SP_EINVAL, SP_ESHAPE (dim odd or < 2). */
enum { SP_ROTARY_UNSCALED = 0, SP_ROTARY_LINEAR = 1, SP_ROTARY_NTK = 2, SP_ROTARY_PARTS = 3 };
int sp_rotary_frequencies(int32_t dim, double base, int32_t scaling, double factor, double trained,
                          double* frequencies_host, float* factor_host);

/* Rotates the first dim elements of every head of every token: pair i, (a, b), becomes
 *     (a cos t - b sin t, b cos t + a sin t) * factor,   t = position * frequencies[i]
 * with the angle formed and reduced in 64 bits, the rest in fp32, rounded once to dtype.  SP_ROTARY_HALF: pair i is elements i and
 * dim / 2 + i; SP_ROTARY_INTERLEAVED: elements 2 i and 2 i + 1.  Elements dim..width are copied.
 *   x, out       [tokens][heads][width], elements of a head contiguous; out may be x with the same strides (elements from dim on are
 *                then not touched), else the two must not overlap
 *   frequencies  device float64 [dim / 2]
 *   positions    device int32 [tokens], any values; or null, then
 *   cu_seqlens   device int32 [batch + 1]: a token's position is its index in its sequence.  Tokens outside the sequences stay as they were
 * Errors: SP_EINVAL, SP_ESHAPE, SP_EHIP. */
enum { SP_ROTARY_HALF = 0, SP_ROTARY_INTERLEAVED = 1 };
int sp_rotary(const void* x, int64_t x_token, int64_t x_head, void* out, int64_t out_token, int64_t out_head,
              int32_t dtype, int32_t tokens, int32_t heads, int32_t width, int32_t dim, int32_t layout,
              const double* frequencies, float factor, const int32_t* positions, const int32_t* cu_seqlens,
              int32_t batch, void* hip_stream);

/* ---- attention --------------------------------------------------------------------------------------------------
 * Packed sequences: sequence b has queries cu_q[b] .. cu_q[b+1] and keys cu_k[b] .. cu_k[b+1] (lengths of zero are fine); query row r
 * of it stands at position i = q_first[b] + r among its keys, j = 0 .. .  With d = j - i, and query head h reading
 * key head h / (heads / kv_heads):
 *     s = scale q.k;   cap > 0: s = cap tanh(s / cap);   slopes: s -= slopes[h] |d|;   bias: s += bias[h][clip(d, -reach, reach) + reach]
 *     out = sum_j softmax_j(s) v_j,   lse = ln sum_j exp(s)          over the visible j
 * j is visible where (-left <= d <= right, a negative bound being none, or j < prefix[b]) and, with documents, doc_q = doc_k >= 0.
 * A bias of minus infinity hides a key too (finite ones below -2e38 weigh like -2e38); positions beyond +-2^30 count as that.  A query
 * that sees nothing gets zeros and lse = minus infinity; one that holds a NaN and sees a key, or sees one whose bias is NaN, gets NaN in
 * both.  Sums and statistics are fp32; bf16 rounds the probabilities to bf16 before their product with the values, and the result.
 * Keys behind a sequence's end and, with documents, keys of a negative document may hold anything; a visible key of one query must be
 * finite also where the mask hides it from another.
 * Rows of out and lse that belong to no sequence are left as they were.  causal attention is right = 0. */
typedef struct {
    const void *q, *k, *v;      /* [total_q][heads][width], [total_k][kv_heads][width] twice; elements of a head contiguous */
    void* out;                  /* [total_q][heads][width]; none of the inputs */
    float* lse;                 /* [total_q][heads] or null */
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, out_token, out_head;     /* strides; 16-byte multiples, like the pointers */
    const int32_t *cu_q, *cu_k; /* [batch + 1] */
    int32_t dtype, batch, heads, kv_heads, width;       /* heads a multiple of kv_heads; width a multiple of 8 up to 128 */
    int32_t total_q, total_k, max_q, max_k;     /* max_*: upper bounds of the lengths */
    float scale, cap;           /* cap <= 0: none */
    int32_t left, right;
    const int32_t* prefix;      /* [batch] or null */
    const int32_t* q_first;     /* [batch], or null: the queries are the last of the sequence, i = keys - queries + r */
    const int32_t *doc_q, *doc_k;       /* [total_q], [total_k], or both null */
    const float* slopes;        /* [heads] or null */
    const float* bias;          /* [heads][2 reach + 1] or null */
    int32_t reach;
} sp_attention_args;

/* Workspace for a call with these sizes (contents of the arrays are not looked at); 0 where none is needed, and for malformed
 * arguments.  256-byte aligned; may be null where 0. */
size_t sp_attention_workspace_bytes(const sp_attention_args* args);
/* Errors: SP_EINVAL, SP_ESHAPE (also: batch beyond 65535, totals or strides beyond 2^29, token strides of k and v beyond 2^23, total_q *
 * heads beyond 2^30, batch * heads beyond 2^22), SP_ENOMEM, SP_EHIP. */
int sp_attention(const sp_attention_args* args, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SP_OPS_H_ */
