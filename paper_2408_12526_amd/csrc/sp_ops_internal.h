// Launchers of the operators of sp_ops.h, for their C entries and for the forward of students that use them.  They check nothing
// that the entries check.
#pragma once

#include "sp_internal.h"
#include "sp_ops.h"

namespace sp {

// Whether the n0 x n1 rows of `width` elements at strides s0 and s1 share no memory (the stride of a single row does not matter).
inline bool rows_apart(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t width)
{
    if (n0 <= 1 || n1 <= 1) return (n0 <= 1 || s0 >= width) && (n1 <= 1 || s1 >= width);
    return s0 < s1 ? s0 >= width && s1 >= (n0 - 1) * s0 + width : s1 >= width && s0 >= (n1 - 1) * s1 + width;
}

hipError_t launch_rotary(const void* x, int64_t xt, int64_t xh, void* out, int64_t ot, int64_t oh, int dtype, int tokens,
                         int heads, int width, int dim, int layout, const double* freq, float factor, const int32_t* pos,
                         const int32_t* cu, int batch, int groups, int64_t xg, int64_t og, hipStream_t s);     // xg, og: elements from group to group

// codes [rows][c_row]: `width` of them, then zeros up to `padded`
hipError_t launch_quantize_int8(const void* x, int64_t x_row, int dtype, int rows, int width, int8_t* codes, int64_t c_row, int padded,
                                float* scales, hipStream_t s);

// out[t][n] = epilogue(sum_k A[t][k] W[n][k] * a_scales[t] w_scales[n] + bias[n]) for k < groups students, each `_ss` behind the one before.
struct Int8Args {
    const int8_t* A;                    // [tokens][a_row], zero from Kd to a_row (a multiple of 128)
    const float* a_scales;
    const int8_t* W;                    // [N][w_row]
    const float *w_scales, *bias;       // bias may be null
    const void* res;                    // may be null
    void* out;
    int64_t a_row, w_row, res_row, out_row;
    size_t a_ss, as_ss, w_ss, ws_ss, b_ss, res_ss, out_ss;      // bytes
    int tokens, N, Kd, groups;
    void* vt;                           // see launch_gemm_int8_qkv
    int64_t ld_vt;
    size_t vt_ss;
    int n_split;
};
bool linear_int8_fused(int tokens, int Kd);
hipError_t launch_linear_int8_fused(const Int8Args& a, const void* x, int64_t x_row, int dtype, int epilogue, hipStream_t s);
hipError_t launch_gemm_int8(const Int8Args& a, int dtype, int epilogue, hipStream_t s);
// The fused q | k | v projection of students (bf16): bias; channels from n_split on are written transposed, vt[channel - n_split][token], ld_vt
// tokens a row (a multiple of 8, at least `tokens`, which is one as well).
hipError_t launch_gemm_int8_qkv(Int8Args a, int n_split, void* vt, int64_t ld_vt, size_t vt_ss, hipStream_t s);

// `groups` students side by side: elements from one's q, k, v, out, slopes and bias to the next one's (their lse follow one another)
struct AttendGroups {
    int groups;
    int64_t q, k, v, out, slopes, bias;
    bool from_start;                    // without q_first: the queries are the first of their sequence, not the last
};
size_t attend_workspace_bytes(const sp_attention_args& a);
// workspace null: never split over the keys
hipError_t launch_attend(const sp_attention_args& a, const AttendGroups& g, void* workspace, hipStream_t s);

}  // namespace sp
