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
    int c_wide;                         // whether the rows of codes are 16-byte aligned
};

// A wave takes row `row`: units of 16 elements, lane after lane, kept in registers between the maximum and the codes up to R units a
// lane.  Codes to c: `width` of them, then zeros up to `padded`.
template <class E, int R>
__device__ __forceinline__ void quantize_row(const QuantArgs& p, int row, int8_t* c, int padded, float* scale_to)
{
    constexpr int PER = 16 / sizeof(E);                     // elements of a 16-byte load
    typedef E Vec __attribute__((ext_vector_type(PER), aligned(sizeof(E))));    // (rows may start anywhere: the hardware takes such loads)
    const int lane = threadIdx.x & 63;
    const E* x = (const E*)(p.x + row * p.x_row);
    const int units = (p.width + 15) >> 4;
    auto fetch = [&](int u, E (&v)[16]) {
        if (u * 16 + 16 <= p.width) {
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
    auto raise = [&](const E (&v)[16]) {
#pragma unroll
        for (int e = 0; e < 16; ++e) { const unsigned m = magnitude(v[e]); most = most > m ? most : m; }
    };
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (lane + 64 * i < units) fetch(lane + 64 * i, kept[i]);
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (lane + 64 * i < units) raise(kept[i]);
    for (int u = lane + 64 * R; u < units; u += 64) {
        E v[16];
        fetch(u, v);
        raise(v);
    }
    most = wave_max_bits(most);
    float scale, factor;
    row_scale(most, scale, factor);
    if (lane == 0) *scale_to = scale;
    // (a factor of zero: the row's codes are zero whatever it holds)
    auto put = [&](int u, const E (&v)[16]) {
        if (p.c_wide && u * 16 + 16 <= padded) {
            v4i w = {0, 0, 0, 0};
            if (factor > 0.f)
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e >> 2] |= (code_of(v[e], factor) & 255) << 8 * (e & 3);
            *(v4i*)(c + u * 16) = w;
        } else {
            for (int e = 0; e < 16; ++e)
                if (u * 16 + e < padded) c[u * 16 + e] = factor > 0.f ? (int8_t)code_of(v[e], factor) : (int8_t)0;
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
    for (int u = units + lane; u * 16 < padded; u += 64) {
        const E none[16] = {};
        put(u, none);
    }
}

template <class E>
__global__ __launch_bounds__(256) void quantize_kernel(QuantArgs p)
{
    const int row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row < p.rows) quantize_row<E, 4>(p, row, p.codes + row * p.c_row, p.padded, p.scales + row);
}

// ---- the product --------------------------------------------------------------------------------------------------

constexpr int kEpiQkv = 3;                                  // see launch_gemm_int8_qkv

// A result from its sum: (float)sum is off by half a step at most, as is every operation behind it.  GELU keeps NaN (a scale of NaN is what the
// quantiser makes of a row that holds one) and infinity: the maximum is the instruction that hands a NaN on, where a median of three drops it.
template <int EPI>
__device__ __forceinline__ float finish(int sum, float scale, float bias, float res)
{
    float y = __builtin_fmaf((float)sum, scale, bias);
    if (EPI == SP_LINEAR_GELU) y = gelu_erf_from(y, __builtin_elementwise_maximum(y, 0.f));
    if (EPI == SP_LINEAR_RESIDUAL) y += res;
    return y;
}

struct Tile {
    int mtiles, ntiles, total, group;   // group: rows of tiles that are gone through together
};

// A workgroup of 2 x 2 waves computes 64 TM tokens x 64 TN channels, a wave TM x TN blocks of 32 x 32 by v_mfma_i32_32x32x32_i8.  Both
// operands come by direct-to-LDS loads in k-tiles of 64 codes, through a ring of `stages` of them.  Rows of four 16-byte slots; slot s of
// row r holds chunk s ^ ((r >> 2) & 3) (no bank conflicts).  Rows behind the last token or channel repeat it; chunks behind the last of a
// weight row repeat that one, against zeros in the activations.
// A k-tile is two steps of 32 codes; a step's fragments are read between the products of the one before.  Behind the first products of the
// second step the next k-tile is waited for, and the one `stages` on is requested, between the others, into the stage that is free then.
// What bounds it: a trip to the L2 and back takes about 2000 cycles, in which a compute unit at full rate multiplies two k-tiles of a 256 x
// 256 tile or eight of a 128 x 128 one: hence the ring, 96 KB of requests under way on a compute unit.
constexpr int ring_stages(int blocks) { return blocks >= 16 ? 4 : blocks >= 4 ? 5 : 8; }
template <int TM, int TN, class E, int EPI>
__global__ __launch_bounds__(256, TM * TN >= 16 ? 1 : 2) void gemm_int8_kernel(Int8Args p, Tile t)
{
    constexpr int BM = 64 * TM, BN = 64 * TN, STAGE = (BM + BN) * 4, NS = ring_stages(TM * TN);     // (16-byte units)
    extern __shared__ uint4 smem[];
    const int chunk = (t.total + 7) >> 3;
    const int lin = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= chunk || lin >= t.total) return;
    // Tiles of an XCD run down a group of token tiles channel by channel: the weights of a tile column and the group's tokens stay in its L2.
    const int tiles = t.mtiles * t.ntiles, m = lin / tiles, tl = lin - m * tiles;
    const int gi = tl / (t.group * t.ntiles), rb = tl - gi * t.group * t.ntiles;
    const int ge = t.mtiles - gi * t.group < t.group ? t.mtiles - gi * t.group : t.group;
    const int nt = rb / ge, mt = gi * t.group + rb % ge;
    const int m0 = mt * BM, n0 = nt * BN;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j31 = lane & 31, g = lane >> 5, wm = wave & 1, wn = wave >> 1;
    const int8_t* A = p.A + (size_t)m * p.a_ss + (size_t)m0 * p.a_row;
    const int8_t* W = p.W + (size_t)m * p.w_ss + (size_t)n0 * p.w_row;
    const int nk = (p.Kd + 63) >> 6, last = (p.Kd - 1) & ~15;

    constexpr int LA = BM / 64, LW = BN / 64;               // wave-loads (16 rows) of a k-tile per wave
    int aoff[LA], woff[LW];
    const int chunk16 = ((lane & 3) ^ (lane >> 4 & 3)) * 16;        // (the same for all of a lane's rows)
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int r = 16 * (wave + 4 * i) + (lane >> 2), rr = m0 + r < p.tokens ? r : p.tokens - 1 - m0;
        aoff[i] = rr * (int)p.a_row + chunk16;
    }
#pragma unroll
    for (int i = 0; i < LW; ++i) {
        const int r = 16 * (wave + 4 * i) + (lane >> 2), rr = n0 + r < p.N ? r : p.N - 1 - n0;
        woff[i] = rr * (int)p.w_row;
    }
    // wave-loads [i0, i1) of the wave's share of a k-tile: tokens, then channels
    auto dma = [&](int kt, int stage, int i0, int i1) {
        uint4* to = smem + stage * STAGE;
        const int k = kt * 64 + chunk16, kw = k < last ? k : last;
#pragma unroll
        for (int i = i0; i < i1; ++i) {
            if (i < LA) load_lds16(A, (lds_void*)(to + (wave + 4 * i) * 64), aoff[i], kt * 64);
            else load_lds16(W, (lds_void*)(to + BM * 4 + (wave + 4 * (i - LA)) * 64), woff[i - LA] + kw, 0);
        }
    };
    i32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    const int row = j31 * 4, key = (j31 >> 2) & 3;
    v4i fa[2][TM], fw[2][TN];
    // fragments [i0, i1) of a step: tokens, then channels
    auto frags = [&](int stage, int s, int i0, int i1) {
        const v4i* a = (const v4i*)(smem + stage * STAGE + wm * TM * 128) + row + ((2 * s + g) ^ key);
        const v4i* w = (const v4i*)(smem + stage * STAGE + BM * 4 + wn * TN * 128) + row + ((2 * s + g) ^ key);
#pragma unroll
        for (int i = i0; i < i1; ++i) {
            if (i < TM) fa[s][i] = a[i * 128];
            else fw[s][i - TM] = w[(i - TM) * 128];
        }
    };
    auto multiply = [&](int s, int i) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[s][i], fa[s][j], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int NL = LA + LW, NF = TM + TN, UNDER_WAY = (NS - 2) * NL;
    for (int kt = 0; kt < NS && kt < nk; ++kt) dma(kt, kt, 0, NL);
    if (nk >= NS) wait_vmcnt<(NS - 1) * NL>();
    else wait_vmcnt<0>();
    barrier_lds();
    frags(0, 0, 0, NF);
    int cur = 0;
    for (int kt = 0; kt < nk; ++kt) {
        const int next = cur + 1 == NS ? 0 : cur + 1;
        const bool more = kt + NS < nk;
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            multiply(0, i);
            frags(cur, 1, i * NF / TN, (i + 1) * NF / TN);
        }
        multiply(1, 0);
        if (kt + 1 < nk) {
            if (kt + NS <= nk) wait_vmcnt<UNDER_WAY>();     // (k-tiles kt + 2 .. kt + NS - 1 have been requested since)
            else wait_vmcnt<0>();
            barrier_lds();                                  // (everybody's fragments of this stage are in registers)
        }
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            if (i > 0) multiply(1, i);
            frags(next, 0, i * NF / TN, (i + 1) * NF / TN); // (behind the last k-tile: of an old one, for nothing)
            if (more) dma(kt + NS, cur, i * NL / TN, (i + 1) * NL / TN);
        }
        cur = next;
    }

    // ---- epilogue: the sums of half the tokens at a time go through LDS as they are, [token][channel], 16-byte chunk c of a row in slot
    // c ^ (token % 32), and leave as whole pieces of rows.  Accumulator element v of lane l: token l % 32, channel 8 (v / 4) + 4 (l / 32) + v % 4.
    const float* sa = (const float*)((const char*)p.a_scales + m * p.as_ss);
    const float* sw = (const float*)((const char*)p.w_scales + m * p.ws_ss);
    const float* bs = p.bias ? (const float*)((const char*)p.bias + m * p.b_ss) : nullptr;
    const E* res = (const E*)((const char*)p.res + m * p.res_ss);
    E* out = (E*)((char*)p.out + m * p.out_ss);
    constexpr int PER = 16 / sizeof(E), TPR = BN / PER, RPI = 256 / TPR, SWZ = BN / 4 < 32 ? BN / 4 - 1 : 31;
    typedef E Vec __attribute__((ext_vector_type(PER), aligned(sizeof(E))));    // (rows may start anywhere)
    const int cc = tid % TPR, n = n0 + cc * PER;
    float ws[PER], bias[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        ws[e] = n + e < p.N ? sw[n + e] : 0.f;
        bias[e] = bs && n + e < p.N ? bs[n + e] : 0.f;
    }
    v4i* stage = (v4i*)smem;
    constexpr int ITER = BM / 2 / RPI;
    const bool whole = n + PER <= p.N;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        // scales and residual of all the thread's rows are requested before anything is waited for (rows behind the last repeat it)
        float st[ITER];
        Vec r[ITER];
        const int x0 = half * (BM / 2) + tid / TPR;
#pragma unroll
        for (int q = 0; q < ITER; ++q) {
            int tok = m0 + x0 + q * RPI;
            tok = tok < p.tokens ? tok : p.tokens - 1;
            st[q] = sa[tok];
            if (EPI == SP_LINEAR_RESIDUAL && whole) r[q] = *(const Vec*)(res + tok * p.res_row + n);
        }
        barrier_lds();                                      // (what stands in the stages is read no more)
        if (wm == half)
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int i = 0; i < TN; ++i)
#pragma unroll
                    for (int v4 = 0; v4 < 4; ++v4) {
                        const int tok = j * 32 + j31, c = (wn * TN + i) * 8 + 2 * v4 + g;
                        stage[tok * (BN / 4) + (c ^ (tok & SWZ))] = v4i{acc[i][j][4 * v4], acc[i][j][4 * v4 + 1], acc[i][j][4 * v4 + 2], acc[i][j][4 * v4 + 3]};
                    }
        barrier_lds();
#pragma unroll
        for (int q = 0; q < ITER; ++q) {
            const int x = tid / TPR + q * RPI, tok = m0 + x0 + q * RPI;
            if (tok >= p.tokens) continue;
            int sum[PER];
#pragma unroll
            for (int c = 0; c < PER / 4; ++c) {
                const v4i a = stage[x * (BN / 4) + ((cc * (PER / 4) + c) ^ (x & SWZ))];
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[c * 4 + e] = a[e];
            }
            if (EPI == kEpiQkv && n >= p.n_split) continue;  // (n_split is a multiple of 8)
            E* to = out + tok * p.out_row + n;
            if (whole) {
                Vec y;
#pragma unroll
                for (int e = 0; e < PER; ++e) y[e] = (E)finish<EPI>(sum[e], st[q] * ws[e], bias[e], EPI == SP_LINEAR_RESIDUAL ? (float)r[q][e] : 0.f);
                *(Vec*)to = y;
            } else {
                const E* from = res + tok * p.res_row + n;
#pragma unroll
                for (int e = 0; e < PER; ++e)
                    if (n + e < p.N) to[e] = (E)finish<EPI>(sum[e], st[q] * ws[e], bias[e], EPI == SP_LINEAR_RESIDUAL ? (float)from[e] : 0.f);
            }
        }
        if constexpr (EPI == kEpiQkv) {
            // channels of the value projection: a thread takes eight tokens of one, sixteen bytes of its row in vt
            constexpr int TG = BM / 16;                     // groups of eight tokens in half a tile
            for (int x = tid; x < BN * TG; x += 256) {
                const int ch = x / TG, n1 = n0 + ch, t0 = x % TG * 8, tok = m0 + half * (BM / 2) + t0;
                if (n1 < p.n_split || n1 >= p.N || tok >= p.tokens) continue;       // (tokens is a multiple of 8)
                const float w1 = sw[n1], b1 = bs ? bs[n1] : 0.f;
                bf16x8 y;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = t0 + e;
                    y[e] = (bf16)finish<EPI>(stage[t * (BN / 4) + ((ch >> 2) ^ (t & SWZ))][ch & 3], sa[tok + e] * w1, b1, 0.f);
                }
                *(bf16x8*)((bf16*)((char*)p.vt + m * p.vt_ss) + (int64_t)(n1 - p.n_split) * p.ld_vt + tok) = y;
            }
        }
    }
}

template <int TM, int TN, class E, int EPI>
hipError_t launch_tile(const Int8Args& a, hipStream_t s)
{
    constexpr size_t smem = (size_t)ring_stages(TM * TN) * (64 * TM + 64 * TN) * 64;
    static_assert(32 * TM * 64 * TN * 4 <= smem, "half the tile's sums go through the stages");
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
    t.group = 16 / TM;                                      // (a thousand tokens)
    hipLaunchKernelGGL(kern, dim3((unsigned)((t.total + 7) / 8 * 8)), dim3(256), smem, s, a, t);
    return hipGetLastError();
}

// ---- few tokens ---------------------------------------------------------------------------------------------------

// Up to 16 TB tokens of one group: a workgroup takes 16 channels, its four waves the k-tiles of 128 codes in turn, straight from memory to the registers
// (v_mfma_i32_16x16x64_i8; a row's 64 contiguous bytes per load), and adds the waves' sums at the end.  What counts is the time of one trip
// to memory: four k-tiles are requested at a time.  FUSED (TB = 1): the workgroup quantises the rows itself, into LDS, while its weights are
// under way; one launch instead of two.
constexpr size_t kFusedBytes = 64 * 1024;                   // codes in LDS
inline size_t fused_pitch(int Kd) { return ((size_t)Kd + 127) / 128 * 128 + 16; }      // (rows start in different banks)

struct FewArgs {
    QuantArgs q;
    int pitch;
};

template <int TB, bool FUSED, class E, int EPI>
__global__ __launch_bounds__(256) void few_int8_kernel(Int8Args p, FewArgs f)
{
    extern __shared__ uint4 smem[];
    __shared__ int sums[4][TB][256];
    __shared__ float scales[16];
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l15 = lane & 15, kq = lane >> 4;
    const int n0 = blockIdx.x * 16, nk = (p.Kd + 127) >> 7, last = (p.Kd - 1) & ~15;
    const int8_t* W = p.W + (size_t)(n0 + l15 < p.N ? n0 + l15 : p.N - 1) * p.w_row;
    constexpr int AHEAD = TB == 4 ? 2 : 4;
    v4i w[AHEAD][2], a[AHEAD][2][TB];
    auto load_w = [&](int i, int kt) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int k = kt * 128 + s * 64 + kq * 16;
            w[i][s] = *(const v4i*)(W + (k < last ? k : last));
        }
    };
    auto load_a = [&](int i, int kt) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int b = 0; b < TB; ++b) {
                const int tok = b * 16 + l15, k = kt * 128 + s * 64 + kq * 16;
                if (FUSED) a[i][s][b] = *(const v4i*)((const char*)smem + (size_t)tok * f.pitch + k);
                else a[i][s][b] = *(const v4i*)(p.A + (size_t)(tok < p.tokens ? tok : p.tokens - 1) * p.a_row + k);
            }
    };
    i32x4 acc[TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) acc[b] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (wave + 4 * i < nk) load_w(i, wave + 4 * i);
    if (FUSED) {
        for (int r = wave; r < p.tokens; r += 4) quantize_row<E, 4>(f.q, r, (int8_t*)smem + (size_t)r * f.pitch, nk * 128, scales + r);
        barrier_lds();
    }
    for (int k0 = wave; k0 < nk; k0 += 4 * AHEAD) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (k0 + 4 * i < nk) load_a(i, k0 + 4 * i);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (k0 + 4 * i < nk) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int b = 0; b < TB; ++b) acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i][s], a[i][s][b], acc[b], 0, 0, 0);
                if (k0 + 4 * (i + AHEAD) < nk) load_w(i, k0 + 4 * (i + AHEAD));
            }
        }
    }
    // element v of lane l: token l % 16, channel 4 (l / 16) + v
#pragma unroll
    for (int b = 0; b < TB; ++b) *(i32x4*)&sums[wave][b][l15 * 16 + kq * 4] = acc[b];
    barrier_lds();
    const int n = n0 + (tid & 15);
    if (n >= p.N) return;
    const float sw = p.w_scales[n], bias = p.bias ? p.bias[n] : 0.f;
#pragma unroll
    for (int b = 0; b < TB; ++b) {
        const int tok = b * 16 + (tid >> 4);
        if (tok >= p.tokens) break;
        const int sum = sums[0][b][tid] + sums[1][b][tid] + sums[2][b][tid] + sums[3][b][tid];
        const float st = FUSED ? scales[tok] : p.a_scales[tok];
        const float res = EPI == SP_LINEAR_RESIDUAL ? (float)((const E*)p.res)[tok * p.res_row + n] : 0.f;
        ((E*)p.out)[tok * p.out_row + n] = (E)finish<EPI>(sum, st * sw, bias, res);
    }
}

template <int TB, bool FUSED, class E, int EPI>
hipError_t launch_few(const Int8Args& a, const QuantArgs& q, hipStream_t s)
{
    const FewArgs f{q, (int)fused_pitch(a.Kd)};
    const size_t smem = FUSED ? 16 * fused_pitch(a.Kd) : 0;
    auto kern = few_int8_kernel<TB, FUSED, E, EPI>;
    if (smem > 32 * 1024) {
        static std::atomic<bool> raised{false};
        if (!raised.load(std::memory_order_acquire)) {
            const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(kFusedBytes + 4096));
            if (e != hipSuccess) return e;
            raised.store(true, std::memory_order_release);
        }
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)((a.N + 15) / 16)), dim3(256), smem, s, a, f);
    return hipGetLastError();
}

// ---- dispatch -----------------------------------------------------------------------------------------------------

// Few tokens: workgroups of 16, 32 or 64 of them, the smallest number that holds them all, where tiles wait for whole trips to memory behind one
// another.  us a call in a graph, 16 / 32 / 64 tokens a workgroup / tiles, by tokens: 1024 -> 4096 channels: 8 5.7 / 5.8 / 6.0 / 8.6, 16 5.7 / 5.8 / 6.2 / 8.6,
// 32 - / 6.3 / 6.7 / 8.6, 64 - / - / 7.7 / 9.1; 768 -> 2304: 16 5.5 / 5.6 / 5.8 / 7.9, 64 7.1 / 8.5; 4096 -> 1024: 16 9.7 / 10.3 / 11.5 / 18.3, 32 11.7 / 12.7 / 18.5,
// 64 15.8 / 19.0.
constexpr int kFewTokens = 64;

template <class E, int EPI>
hipError_t launch_tiles(const Int8Args& a, hipStream_t s)
{
    // Tile: rounds of tiles over the compute units, each at a price of so many us and so many for a k-tile of 64 codes (two workgroups of
    // the smaller ones share a unit, so that one's stores run while the other multiplies; the large one has it to itself).  us a call with the
    // quantiser, residual, tiles of 64 / 128 / 256 a side, by tokens: 4096 -> 1024 channels: 1024 23.5 / 33.7 / 65, 2048 30 / 36 / 66, 4096 51 / 42 / 72, 8192 93 / 73 /
    // 81, 14722 176 / 130 / 106; 1024 -> 4096: 256 13.3 / 15 / 28, 1024 21 / 18 / 30, 2048 35 / 24 / 33, 4096 63 / 42 / 39, 8192 117 / 78 / 71, 14722 212 / 142 / 132;
    // 768 -> 2304: 4096 36 / 31 / 31, 8192 65 / 46 / 58, 14722 110 / 72 / 83.
    const double nk = (a.Kd + 63) / 64;
    auto cost = [&](int side, double fixed, double each) {
        const int64_t tiles = (int64_t)((a.tokens + side - 1) / side) * ((a.N + side - 1) / side) * a.groups;
        return (double)((tiles + 255) / 256) * (fixed + each * nk);
    };
    const double c64 = cost(64, 2, 0.125), c128 = cost(128, 2, 0.33), c256 = cost(256, 10, 1);
    if (c256 <= c128 && c256 <= c64) return launch_tile<4, 4, E, EPI>(a, s);
    return c128 <= c64 ? launch_tile<2, 2, E, EPI>(a, s) : launch_tile<1, 1, E, EPI>(a, s);
}

template <class E, int EPI>
hipError_t launch_epilogue(const Int8Args& a, hipStream_t s)
{
    // (students side by side come with at least 2048 rows each)
    if (a.tokens > kFewTokens || a.groups > 1) return launch_tiles<E, EPI>(a, s);
    if (a.tokens <= 16) return launch_few<1, false, E, EPI>(a, QuantArgs{}, s);
    if (a.tokens <= 32) return launch_few<2, false, E, EPI>(a, QuantArgs{}, s);
    return launch_few<4, false, E, EPI>(a, QuantArgs{}, s);
}

template <class E>
hipError_t launch_type(const Int8Args& a, int epilogue, hipStream_t s)
{
    switch (epilogue) {
        case SP_LINEAR_GELU: return launch_epilogue<E, SP_LINEAR_GELU>(a, s);
        case SP_LINEAR_RESIDUAL: return launch_epilogue<E, SP_LINEAR_RESIDUAL>(a, s);
        default: return launch_epilogue<E, SP_LINEAR_PLAIN>(a, s);
    }
}

template <class E>
hipError_t launch_fused_type(const Int8Args& a, const QuantArgs& q, int epilogue, hipStream_t s)
{
    switch (epilogue) {
        case SP_LINEAR_GELU: return launch_few<1, true, E, SP_LINEAR_GELU>(a, q, s);
        case SP_LINEAR_RESIDUAL: return launch_few<1, true, E, SP_LINEAR_RESIDUAL>(a, q, s);
        default: return launch_few<1, true, E, SP_LINEAR_PLAIN>(a, q, s);
    }
}

}  // namespace

hipError_t launch_gemm_int8(const Int8Args& a, int dtype, int epilogue, hipStream_t s)
{
    return dtype == SP_DTYPE_FP32 ? launch_type<float>(a, epilogue, s) : launch_type<bf16>(a, epilogue, s);
}

hipError_t launch_gemm_int8_qkv(Int8Args a, int n_split, void* vt, int64_t ld_vt, size_t vt_ss, hipStream_t s)
{
    if (a.tokens % 8 || n_split % 8 || ld_vt % 8 || ((uintptr_t)vt & 15) || (vt_ss & 15)) return hipErrorInvalidValue;
    a.n_split = n_split;
    a.vt = vt;
    a.ld_vt = ld_vt;
    a.vt_ss = vt_ss;
    return launch_tiles<bf16, kEpiQkv>(a, s);
}

static QuantArgs quant_args(const void* x, int64_t x_row, int dtype, int rows, int width, int8_t* codes, int64_t c_row, int padded, float* scales)
{
    const size_t row = (size_t)(x_row * (dtype == SP_DTYPE_FP32 ? 4 : 2));
    return QuantArgs{(const char*)x, row, codes, (size_t)c_row, scales, rows, width, padded,
                     !(((uintptr_t)codes | (size_t)c_row) & 15)};
}

hipError_t launch_quantize_int8(const void* x, int64_t x_row, int dtype, int rows, int width, int8_t* codes, int64_t c_row, int padded,
                                float* scales, hipStream_t s)
{
    const QuantArgs a = quant_args(x, x_row, dtype, rows, width, codes, c_row, padded, scales);
    const dim3 grid((unsigned)((a.rows + 3) / 4));
    if (dtype == SP_DTYPE_FP32) hipLaunchKernelGGL(quantize_kernel<float>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(quantize_kernel<bf16>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

// Rows quantised in the product's own launch: one launch less, but every workgroup does it again.  us a call, in one launch / two, by tokens: eager
// calls, where the second launch is the host's, 768 -> 2304 9.6 / 11.8 from 1 to 16, 4096 -> 1024 9.2 / 11.4, 16 13.5 / 11.4; in a graph 768 -> 2304 1 4.6 / 4.9,
// 8 5.9 / 5.3, 16 7.9 / 5.5, 4096 -> 1024 1 6.8 / 8.0, 8 9.2 / 9.0, 16 13.5 / 9.7.
bool linear_int8_fused(int tokens, int Kd) { return tokens <= 16 && 16 * fused_pitch(Kd) <= kFusedBytes + 4096; }

hipError_t launch_linear_int8_fused(const Int8Args& a, const void* x, int64_t x_row, int dtype, int epilogue, hipStream_t s)
{
    const QuantArgs q = quant_args(x, x_row, dtype, a.tokens, a.Kd, nullptr, 0, 0, nullptr);
    return dtype == SP_DTYPE_FP32 ? launch_fused_type<float>(a, q, epilogue, s) : launch_fused_type<bf16>(a, q, epilogue, s);
}

}  // namespace sp

using namespace sp;

namespace {

constexpr int32_t kMostRows = (1 << 26) - 4;                // a wave each, and a grid has fewer than 2^32 threads
constexpr int32_t kMostWidth = INT32_MAX - 2048;            // (a wave forms the offsets of 64 units of 16 elements behind a row's last one)
constexpr int32_t kMostWidthIn = 131072;                    // 131072 * 127 * 127 < 2^31
size_t codes_row(int32_t width_in) { return ((size_t)width_in + 127) / 128 * 128; }
size_t codes_bytes(int32_t tokens, int32_t width_in) { return ((size_t)tokens * codes_row(width_in) + 255) / 256 * 256; }

}  // namespace

extern "C" {

int sp_quantize_int8(const void* x, int64_t x_row, int32_t dtype, int32_t rows, int32_t width, int8_t* codes, int64_t c_row,
                     float* scales, void* hip_stream)
{
    if (dtype != SP_DTYPE_FP32 && dtype != SP_DTYPE_BF16) return SP_EINVAL;
    if (rows < 0 || rows > kMostRows || width < 1 || width > kMostWidth || (rows > 1 && (x_row < 0 || c_row < width))) return SP_ESHAPE;
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
    if (w_row < width_in || w_row % 16 || w_row > (1 << 20) || width_out > (1 << 24) || tokens > kMostRows) return SP_ESHAPE;
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
    Int8Args a{};
    a.A = codes; a.a_scales = scales; a.W = w_codes; a.w_scales = w_scales; a.bias = bias; a.res = residual; a.out = out;
    a.a_row = (int64_t)row; a.w_row = w_row; a.res_row = residual_row; a.out_row = out_row;
    a.tokens = tokens; a.N = width_out; a.Kd = width_in; a.groups = 1;
    if (linear_int8_fused(tokens, width_in)) return launch_linear_int8_fused(a, x, x_row, dtype, epilogue, s) == hipSuccess ? SP_OK : SP_EHIP;
    if (launch_quantize_int8(x, x_row, dtype, tokens, width_in, codes, (int64_t)row, (int)row, scales, s) != hipSuccess) return SP_EHIP;
    return launch_gemm_int8(a, dtype, epilogue, s) == hipSuccess ? SP_OK : SP_EHIP;
}

}  // extern "C"
