// Products in 8-bit integers with a scale for each token and each output channel:
//   out[t][n] = epilogue((c[t] . w[n]) * s[t] sw[n] + bias[n]),   c[t], s[t] the codes and the scale of the row x[t]
// The sum over the reduction is exact (32-bit integers hold 131072 products of codes); everything behind it is fp32.
#include <atomic>

#include "sp_ops_internal.h"

namespace sp {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// ---- rows to codes ------------------------------------------------------------------------------------------------

__device__ __forceinline__ unsigned wave_max_bits(unsigned v)      // of magnitudes: the order of their bits is theirs, NaN above infinity
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const unsigned o = __shfl_xor(v, d);
        v = v > o ? v : o;
    }
    return v;
}

template <class E>
__device__ __forceinline__ unsigned magnitude(E v) { return __builtin_bit_cast(unsigned, (float)v) & 0x7fffffffu; }

// Scale and factor of a row by its largest magnitude (bits).
__device__ __forceinline__ void row_scale(unsigned bits, float& scale, float& factor)
{
    const float a = __builtin_bit_cast(float, bits);
    if (bits >= 0x7f800000u) {                              // an infinity or a NaN in the row
        scale = __builtin_nanf("");
        factor = 0.f;
    } else if (a < 0x1p-100f) {                             // (127 / a stays finite above)
        scale = factor = 0.f;
    } else {
        scale = a / 127.f;
        factor = 127.f / a;
    }
}
template <class E>
__device__ __forceinline__ int code_of(E v, float factor) { return (int)__builtin_rintf((float)v * factor); }

struct QuantArgs {
    const char* x;
    size_t x_row;                       // bytes
    int8_t* codes;
    size_t c_row;
    float* scales;
    int rows, width, padded;
};

// A wave takes a row: units of 16 elements, lane after lane, kept in registers between the maximum and the codes up to R units a
// lane.  WIDE: rows and codes are 16-byte aligned.
template <class E, bool WIDE, int R>
__global__ __launch_bounds__(256) void quantize_kernel(QuantArgs p)
{
    constexpr int PER = 16 / sizeof(E);                     // elements of a 16-byte load
    typedef E Vec __attribute__((ext_vector_type(PER)));
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= p.rows) return;
    const E* x = (const E*)(p.x + row * p.x_row);
    int8_t* c = p.codes + row * p.c_row;
    const int units = (p.width + 15) >> 4;
    auto fetch = [&](int u, E (&v)[16]) {
        if (WIDE && u * 16 + 16 <= p.width) {
#pragma unroll
            for (int i = 0; i < 16 / PER; ++i) {
                const Vec w = ((const Vec*)(x + u * 16))[i];
#pragma unroll
                for (int e = 0; e < PER; ++e) v[i * PER + e] = w[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = u * 16 + e < p.width ? x[u * 16 + e] : (E)0.f;
        }
    };
    E kept[R][16];
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int u = lane + 64 * i;
        if (u < units) {
            fetch(u, kept[i]);
#pragma unroll
            for (int e = 0; e < 16; ++e) { const unsigned m = magnitude(kept[i][e]); most = most > m ? most : m; }
        }
    }
    for (int u = lane + 64 * R; u < units; u += 64) {
        E v[16];
        fetch(u, v);
#pragma unroll
        for (int e = 0; e < 16; ++e) { const unsigned m = magnitude(v[e]); most = most > m ? most : m; }
    }
    most = wave_max_bits(most);
    float scale, factor;
    row_scale(most, scale, factor);
    if (lane == 0) p.scales[row] = scale;
    // (a factor of zero: the row's codes are zero whatever it holds)
    auto put = [&](int u, const E (&v)[16]) {
        if (WIDE && u * 16 + 16 <= p.padded) {
            v4i w = {0, 0, 0, 0};
            if (factor > 0.f)
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e >> 2] |= (code_of(v[e], factor) & 255) << 8 * (e & 3);
            *(v4i*)(c + u * 16) = w;
        } else {
            for (int e = 0; e < 16; ++e)
                if (u * 16 + e < p.padded) c[u * 16 + e] = factor > 0.f ? (int8_t)code_of(v[e], factor) : (int8_t)0;
        }
    };
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (lane + 64 * i < units) put(lane + 64 * i, kept[i]);
    for (int u = lane + 64 * R; u < units; u += 64) {
        E v[16];
        fetch(u, v);
        put(u, v);
    }
    for (int u = units + lane; u * 16 < p.padded; u += 64) {
        const E none[16] = {};
        put(u, none);
    }
}

// ---- the product --------------------------------------------------------------------------------------------------

struct Tile {
    int mtiles, ntiles, total;
};

// A workgroup of 2 x 2 waves computes 64 TM tokens x 64 TN channels, a wave TM x TN blocks of 32 x 32 by v_mfma_i32_32x32x32_i8.  Both
// operands come by direct-to-LDS loads in k-tiles of 128 codes, two stages: the next k-tile travels while one is multiplied.  Rows of
// eight 16-byte slots; slot s of row r holds chunk s ^ ((r >> 1) & 7) (no bank conflicts).  Rows behind the last token or channel repeat it;
// chunks behind the last of a weight row repeat that one, against zeros in the activations.
template <int TM, int TN, class E, int EPI>
__global__ __launch_bounds__(256) void gemm_int8_kernel(Int8Args p, Tile t)
{
    constexpr int BM = 64 * TM, BN = 64 * TN, STAGE = (BM + BN) * 8;    // 16-byte units
    extern __shared__ uint4 smem[];
    const int chunk = (t.total + 7) >> 3;
    const int lin = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= chunk || lin >= t.total) return;
    const int tiles = t.mtiles * t.ntiles, m = lin / tiles, tl = lin - m * tiles;
    const int mt = tl / t.ntiles, nt = tl - mt * t.ntiles;
    const int m0 = mt * BM, n0 = nt * BN;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j31 = lane & 31, g = lane >> 5, wm = wave & 1, wn = wave >> 1;
    const int8_t* A = p.A + (size_t)m * p.a_ss + (size_t)m0 * p.a_row;
    const int8_t* W = p.W + (size_t)m * p.w_ss + (size_t)n0 * p.w_row;
    const int nk = (p.Kd + 127) >> 7, last = (p.Kd - 1) & ~15;

    int aoff[BM / 32], woff[BN / 32];
    const int wchunk = lane & 7;
#pragma unroll
    for (int i = 0; i < BM / 32; ++i) {
        const int r = 8 * (wave + 4 * i) + (lane >> 3), rr = m0 + r < p.tokens ? r : p.tokens - 1 - m0;
        aoff[i] = rr * (int)p.a_row + (wchunk ^ ((r >> 1) & 7)) * 16;
    }
#pragma unroll
    for (int i = 0; i < BN / 32; ++i) {
        const int r = 8 * (wave + 4 * i) + (lane >> 3), rr = n0 + r < p.N ? r : p.N - 1 - n0;
        woff[i] = rr * (int)p.w_row;
    }
    auto dma = [&](int kt, int stage) {
        uint4* to = smem + stage * STAGE;
#pragma unroll
        for (int i = 0; i < BM / 32; ++i) load_lds16(A, (lds_void*)(to + (wave + 4 * i) * 64), aoff[i], kt * 128);
#pragma unroll
        for (int i = 0; i < BN / 32; ++i) {
            const int r = 8 * (wave + 4 * i) + (lane >> 3), k = kt * 128 + (wchunk ^ ((r >> 1) & 7)) * 16;
            load_lds16(W, (lds_void*)(to + BM * 8 + (wave + 4 * i) * 64), woff[i] + (k < last ? k : last), 0);
        }
    };
    i32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    const int row = j31 * 8, key = (j31 >> 1) & 7;
    dma(0, 0);
    for (int kt = 0; kt < nk; ++kt) {
        wait_vmcnt<0>();
        barrier_lds();                                      // the k-tile is there, and everybody is done with the other stage
        if (kt + 1 < nk) dma(kt + 1, (kt + 1) & 1);
        const v4i* a = (const v4i*)(smem + (kt & 1) * STAGE + wm * TM * 256) + row;
        const v4i* w = (const v4i*)(smem + (kt & 1) * STAGE + BM * 8 + wn * TN * 256) + row;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int c = (2 * s + g) ^ key;
            v4i fa[TM], fw[TN];
#pragma unroll
            for (int j = 0; j < TM; ++j) fa[j] = a[j * 256 + c];
#pragma unroll
            for (int i = 0; i < TN; ++i) fw[i] = w[i * 256 + c];
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[i], fa[j], acc[i][j], 0, 0, 0);
        }
    }
    // Accumulator element v of lane l: token l % 32, channel 8 (v / 4) + 4 (l / 32) + v % 4.
    const float* sa = (const float*)((const char*)p.a_scales + m * p.as_ss);
    const float* sw = (const float*)((const char*)p.w_scales + m * p.ws_ss);
    const float* bs = p.bias ? (const float*)((const char*)p.bias + m * p.b_ss) : nullptr;
    const E* res = (const E*)((const char*)p.res + m * p.res_ss);
    E* out = (E*)((char*)p.out + m * p.out_ss);
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const int tok = m0 + (wm * TM + j) * 32 + j31;
        if (tok >= p.tokens) continue;
        const float st = sa[tok];
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int n = n0 + (wn * TN + i) * 32 + 8 * (v >> 2) + 4 * g + (v & 3);
                if (n >= p.N) continue;
                float y = __builtin_fmaf((float)acc[i][j][v], st * sw[n], bs ? bs[n] : 0.f);
                if (EPI == SP_LINEAR_GELU) y = gelu_erf_fast(y);
                if (EPI == SP_LINEAR_RESIDUAL) y += (float)res[tok * p.res_row + n];
                out[tok * p.out_row + n] = (E)y;
            }
    }
}

template <int TM, int TN, class E, int EPI>
hipError_t launch_tile(const Int8Args& a, hipStream_t s)
{
    constexpr size_t smem = 2 * (64 * TM + 64 * TN) * 128;
    auto kern = gemm_int8_kernel<TM, TN, E, EPI>;
    if (smem > 48 * 1024) {
        static std::atomic<bool> raised{false};             // per instantiation; the attribute is sticky for the process
        if (!raised.load(std::memory_order_acquire)) {
            const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e != hipSuccess) return e;
            raised.store(true, std::memory_order_release);
        }
    }
    Tile t;
    t.mtiles = (a.tokens + 64 * TM - 1) / (64 * TM);
    t.ntiles = (a.N + 64 * TN - 1) / (64 * TN);
    t.total = t.mtiles * t.ntiles * a.groups;
    hipLaunchKernelGGL(kern, dim3((unsigned)((t.total + 7) / 8 * 8)), dim3(256), smem, s, a, t);
    return hipGetLastError();
}

template <class E>
hipError_t launch_type(const Int8Args& a, int epilogue, hipStream_t s)
{
    switch (epilogue) {
        case SP_LINEAR_GELU: return launch_tile<2, 2, E, SP_LINEAR_GELU>(a, s);
        case SP_LINEAR_RESIDUAL: return launch_tile<2, 2, E, SP_LINEAR_RESIDUAL>(a, s);
        default: return launch_tile<2, 2, E, SP_LINEAR_PLAIN>(a, s);
    }
}

template <class E>
hipError_t launch_quantize_type(const QuantArgs& a, hipStream_t s)
{
    const bool wide = !(((uintptr_t)a.x | a.x_row | (uintptr_t)a.codes | a.c_row) & 15);
    const dim3 grid((unsigned)((a.rows + 3) / 4));
    if (wide) hipLaunchKernelGGL((quantize_kernel<E, true, 4>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((quantize_kernel<E, false, 1>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_int8(const Int8Args& a, int dtype, int epilogue, hipStream_t s)
{
    return dtype == SP_DTYPE_FP32 ? launch_type<float>(a, epilogue, s) : launch_type<bf16>(a, epilogue, s);
}

hipError_t launch_quantize_int8(const void* x, int64_t x_row, int dtype, int rows, int width, int8_t* codes, int64_t c_row, int padded,
                                float* scales, hipStream_t s)
{
    const QuantArgs a{(const char*)x, (size_t)(x_row * (dtype == SP_DTYPE_FP32 ? 4 : 2)), codes, (size_t)c_row, scales, rows, width, padded};
    return dtype == SP_DTYPE_FP32 ? launch_quantize_type<float>(a, s) : launch_quantize_type<bf16>(a, s);
}

}  // namespace sp

using namespace sp;

namespace {

constexpr int32_t kMostWidthIn = 131072;                    // 131072 * 127 * 127 < 2^31
size_t codes_row(int32_t width_in) { return ((size_t)width_in + 127) / 128 * 128; }
size_t codes_bytes(int32_t tokens, int32_t width_in) { return ((size_t)tokens * codes_row(width_in) + 255) / 256 * 256; }

}  // namespace

extern "C" {

int sp_quantize_int8(const void* x, int64_t x_row, int32_t dtype, int32_t rows, int32_t width, int8_t* codes, int64_t c_row,
                     float* scales, void* hip_stream)
{
    if (dtype != SP_DTYPE_FP32 && dtype != SP_DTYPE_BF16) return SP_EINVAL;
    if (rows < 0 || width < 1 || width > INT32_MAX - 16 || (rows > 1 && (x_row < 0 || c_row < width))) return SP_ESHAPE;
    if (rows == 0) return SP_OK;
    if (!x || !codes || !scales || ((uintptr_t)x & (dtype == SP_DTYPE_FP32 ? 3 : 1)) || ((uintptr_t)scales & 3)) return SP_EINVAL;
    return launch_quantize_int8(x, x_row, dtype, rows, width, codes, c_row, width, scales, (hipStream_t)hip_stream) == hipSuccess ? SP_OK
                                                                                                                                  : SP_EHIP;
}

size_t sp_linear_int8_workspace_bytes(int32_t tokens, int32_t width_in)
{
    if (tokens < 1 || width_in < 1 || width_in > kMostWidthIn) return 0;
    return codes_bytes(tokens, width_in) + (size_t)tokens * 4;
}

int sp_linear_int8(const void* x, int64_t x_row, int32_t dtype, int32_t tokens, int32_t width_in, const int8_t* w_codes, int64_t w_row,
                   const float* w_scales, int32_t width_out, const float* bias, int32_t epilogue, const void* residual,
                   int64_t residual_row, void* out, int64_t out_row, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (dtype != SP_DTYPE_FP32 && dtype != SP_DTYPE_BF16) return SP_EINVAL;
    if (epilogue < SP_LINEAR_PLAIN || epilogue > SP_LINEAR_RESIDUAL) return SP_EINVAL;
    if (tokens < 0 || width_in < 1 || width_in > kMostWidthIn || width_out < 1) return SP_ESHAPE;
    // (offsets inside a tile of weights are 32-bit; the bounds on the sizes keep numbers of tiles inside 32 bits)
    if (w_row < width_in || w_row % 16 || w_row > (1 << 20) || width_out > (1 << 24) || tokens > (1 << 28)) return SP_ESHAPE;
    if ((int64_t)((tokens + 63) / 64) * ((width_out + 63) / 64) > (1 << 23)) return SP_ESHAPE;
    if (tokens > 1 && (x_row < 0 || out_row < width_out || residual_row < 0)) return SP_ESHAPE;
    if (tokens == 0) return SP_OK;
    const uintptr_t low = dtype == SP_DTYPE_FP32 ? 3 : 1;
    if (!x || !w_codes || !w_scales || !out || !workspace || (epilogue == SP_LINEAR_RESIDUAL) != (residual != nullptr)) return SP_EINVAL;
    if ((((uintptr_t)x | (uintptr_t)out | (uintptr_t)residual) & low) || ((uintptr_t)w_codes & 15) || ((uintptr_t)workspace & 255) ||
        (((uintptr_t)w_scales | (uintptr_t)bias) & 3) || x == out || (out == residual && out_row != residual_row))
        return SP_EINVAL;
    if (workspace_bytes < sp_linear_int8_workspace_bytes(tokens, width_in)) return SP_ENOMEM;
    const size_t row = codes_row(width_in);
    int8_t* codes = (int8_t*)workspace;
    float* scales = (float*)((char*)workspace + codes_bytes(tokens, width_in));
    hipStream_t s = (hipStream_t)hip_stream;
    if (launch_quantize_int8(x, x_row, dtype, tokens, width_in, codes, (int64_t)row, (int)row, scales, s) != hipSuccess) return SP_EHIP;
    Int8Args a{};
    a.A = codes; a.a_scales = scales; a.W = w_codes; a.w_scales = w_scales; a.bias = bias; a.res = residual; a.out = out;
    a.a_row = (int64_t)row; a.w_row = w_row; a.res_row = residual_row; a.out_row = out_row;
    a.tokens = tokens; a.N = width_out; a.Kd = width_in; a.groups = 1;
    return launch_gemm_int8(a, dtype, epilogue, s) == hipSuccess ? SP_OK : SP_EHIP;
}

}  // extern "C"
