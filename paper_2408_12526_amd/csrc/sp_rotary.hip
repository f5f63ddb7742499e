// Rotary positions: the first `dim` elements of every head are turned, pair by pair, by an angle that grows with the token's
// position, so that a query's product with a key depends on their distance alone.
#include <cmath>

#include "sp_ops_internal.h"

namespace sp {

namespace {

struct RotaryArgs {
    const char* x;
    char* out;
    size_t xt, xh, ot, oh, xg, og;      // strides in bytes (token, head, group)
    const double* freq;
    const int32_t *pos, *cu;
    float factor;
    int tokens, heads, width, half, batch, per, copy;   // per: heads a thread takes; copy: whether elements from dim on are copied
    int units, turn_units;              // units of a head: of V pairs, then of 2 V copied elements
};

// (the same instructions whatever V and layout, so that in place and not, and any alignment, give the same bits)
__device__ __forceinline__ void turn(float a, float b, float c, float s, float& ra, float& rb)
{
    ra = __builtin_fmaf(a, c, -(b * s));
    rb = __builtin_fmaf(b, c, a * s);
}

// One thread: V pairs (or 2 V elements behind the rotated ones) of one token, for `per` heads.  The angle is the same for every head:
// its turns are formed in 64 bits, position * (frequency / 2 pi), and reduced there (2^-53 relative: 2^-33 turns off at
// position 2^20), sine and cosine taken in fp32 from the fraction of a turn, once for all the thread's heads.
// Bound by memory: every element read and written once, 16 bytes a lane.
template <class E, int V, int LAYOUT>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs p)
{
    typedef E Vec __attribute__((ext_vector_type(V), aligned(sizeof(E))));      // (heads may start anywhere: the hardware takes such loads)
    const unsigned at = blockIdx.x * 256u + threadIdx.x;
    const int token = (int)(at / (unsigned)p.units), u = (int)(at - (unsigned)token * (unsigned)p.units);
    if (token >= p.tokens) return;
    int position;
    if (p.pos) {
        position = p.pos[token];
    } else {                                                // the last sequence that begins at or before the token
        if (token < p.cu[0] || token >= p.cu[p.batch]) return;
        int lo = 0, hi = p.batch;                           // cu[lo] <= token < cu[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (p.cu[mid] <= token) lo = mid;
            else hi = mid;
        }
        position = token - p.cu[lo];
    }
    const int h0 = blockIdx.y * p.per, h1 = h0 + p.per < p.heads ? h0 + p.per : p.heads;
    const char* x = p.x + token * p.xt + blockIdx.z * p.xg;
    char* out = p.out + token * p.ot + blockIdx.z * p.og;
    if (u >= p.turn_units) {
        if (!p.copy) return;
        int e0 = 2 * p.half + (u - p.turn_units) * 2 * V;
        if (e0 + 2 * V > p.width && p.width - 2 * V >= 2 * p.half) e0 = p.width - 2 * V;    // (the last unit: some elements again)
        const int n = p.width - e0 < 2 * V ? p.width - e0 : 2 * V;
        for (int h = h0; h < h1; ++h) {
            const E* a = (const E*)(x + h * p.xh) + e0;
            E* o = (E*)(out + h * p.oh) + e0;
            if (n == 2 * V) {
                const Vec a0 = ((const Vec*)a)[0], a1 = ((const Vec*)a)[1];
                ((Vec*)o)[0] = a0;
                ((Vec*)o)[1] = a1;
            } else {
                for (int e = 0; e < n; ++e) o[e] = a[e];
            }
        }
        return;
    }
    // (the last unit of a head that is no multiple of V begins earlier and does some pairs again: never in place)
    const int p0 = u * V + V <= p.half ? u * V : p.half - V;
    float cs[V], sn[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        double t = (double)position * (p.freq[p0 + e] * 0.15915494309189533577);    // 1 / 2 pi
        t -= __builtin_rint(t);
        float s, c;
        sincospif((float)(2.0 * t), &s, &c);
        cs[e] = c * p.factor;
        sn[e] = s * p.factor;
    }
    const int ea = LAYOUT == SP_ROTARY_HALF ? p0 : 2 * p0, eb = LAYOUT == SP_ROTARY_HALF ? p.half + p0 : ea + V;
#pragma unroll 4
    for (int h = h0; h < h1; ++h) {
        const Vec a = *(const Vec*)((const E*)(x + h * p.xh) + ea), b = *(const Vec*)((const E*)(x + h * p.xh) + eb);
        Vec ra, rb;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (LAYOUT == SP_ROTARY_HALF) {
                float r0, r1;
                turn((float)a[e], (float)b[e], cs[e], sn[e], r0, r1);
                ra[e] = (E)r0;
                rb[e] = (E)r1;
            } else {                                        // pair e: elements 2 e and 2 e + 1 of the 2 V
                const int i = 2 * e % V;
                const float va = 2 * e < V ? (float)a[i] : (float)b[i], vb = 2 * e + 1 < V ? (float)a[(i + 1) % V] : (float)b[(i + 1) % V];
                float r0, r1;
                turn(va, vb, cs[e], sn[e], r0, r1);
                if (2 * e < V) ra[i] = (E)r0;
                else rb[i] = (E)r0;
                if (2 * e + 1 < V) ra[(i + 1) % V] = (E)r1;
                else rb[(i + 1) % V] = (E)r1;
            }
        }
        *(Vec*)((E*)(out + h * p.oh) + ea) = ra;
        *(Vec*)((E*)(out + h * p.oh) + eb) = rb;
    }
}

template <class E, int V>
hipError_t launch_width(RotaryArgs a, int groups, int layout, hipStream_t s)
{
    a.turn_units = (a.half + V - 1) / V;
    a.units = a.turn_units + (a.copy ? (a.width - 2 * a.half + 2 * V - 1) / (2 * V) : 0);
    const long blocks = ((long)a.tokens * a.units + 255) / 256;
    // Heads of a thread: all of them share its sines, but a launch of few threads is spread over heads as well (four workgroups a
    // compute unit).
    int parts = (int)(1024 / (blocks * groups));
    parts = parts < 1 ? 1 : parts > a.heads ? a.heads : parts;
    a.per = (a.heads + parts - 1) / parts;
    const dim3 grid((unsigned)blocks, (unsigned)((a.heads + a.per - 1) / a.per), (unsigned)groups);
    if (layout == SP_ROTARY_HALF) hipLaunchKernelGGL((rotary_kernel<E, V, SP_ROTARY_HALF>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((rotary_kernel<E, V, SP_ROTARY_INTERLEAVED>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const void* x, int64_t xt, int64_t xh, void* out, int64_t ot, int64_t oh, int dtype, int tokens,
                         int heads, int width, int dim, int layout, const double* freq, float factor, const int32_t* pos,
                         const int32_t* cu, int batch, int groups, int64_t xg, int64_t og, hipStream_t s)
{
    const int sz = dtype == SP_DTYPE_FP32 ? 4 : 2;
    const RotaryArgs a{(const char*)x, (char*)out, (size_t)(xt * sz), (size_t)(xh * sz), (size_t)(ot * sz), (size_t)(oh * sz),
                       (size_t)(xg * sz), (size_t)(og * sz), freq, pos, cu,
                       factor, tokens, heads, width, dim / 2, batch, 0, x != out && width > dim, 0, 0};
    // Pairs of a unit: 16 bytes of each kind, fewer where the head has not as many, and in place where they do not divide it
    int v = 16 / sz;
    while (v > a.half || (x == out && a.half % v)) v >>= 1;
    if (dtype == SP_DTYPE_FP32)
        return v == 4 ? launch_width<float, 4>(a, groups, layout, s) : v == 2 ? launch_width<float, 2>(a, groups, layout, s) : launch_width<float, 1>(a, groups, layout, s);
    switch (v) {
        case 8: return launch_width<bf16, 8>(a, groups, layout, s);
        case 4: return launch_width<bf16, 4>(a, groups, layout, s);
        case 2: return launch_width<bf16, 2>(a, groups, layout, s);
        default: return launch_width<bf16, 1>(a, groups, layout, s);
    }
}

}  // namespace sp

using namespace sp;

extern "C" {

int sp_rotary_frequencies(int32_t dim, double base, int32_t scaling, double factor, double trained, double* f, float* factor_host)
{
    if (!f || !factor_host || scaling < SP_ROTARY_UNSCALED || scaling > SP_ROTARY_PARTS) return SP_EINVAL;
    if (!(base > 1.0) || !std::isfinite(base) || !(factor >= 1.0) || !std::isfinite(factor)) return SP_EINVAL;
    if (scaling == SP_ROTARY_PARTS && (!(trained >= 1.0) || !std::isfinite(trained))) return SP_EINVAL;
    if (dim < 2 || dim % 2 || (scaling == SP_ROTARY_NTK && dim < 4)) return SP_ESHAPE;
    if (scaling == SP_ROTARY_NTK) base *= std::pow(factor, (double)dim / (dim - 2));
    for (int32_t i = 0; i < dim / 2; ++i) {
        double v = std::pow(base, -2.0 * i / dim);
        if (scaling == SP_ROTARY_LINEAR) v /= factor;
        if (scaling == SP_ROTARY_PARTS) {
            double g = (trained * v * 0.15915494309189533577 - 1.0) / 31.0;
            g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
            v = v * g + v / factor * (1.0 - g);
        }
        f[i] = v;
    }
    *factor_host = scaling == SP_ROTARY_PARTS ? (float)(1.0 + 0.1 * std::log(factor)) : 1.f;
    return SP_OK;
}

int sp_rotary(const void* x, int64_t x_token, int64_t x_head, void* out, int64_t out_token, int64_t out_head, int32_t dtype,
              int32_t tokens, int32_t heads, int32_t width, int32_t dim, int32_t layout, const double* frequencies,
              float factor, const int32_t* positions, const int32_t* cu_seqlens, int32_t batch, void* hip_stream)
{
    if (dtype != SP_DTYPE_FP32 && dtype != SP_DTYPE_BF16) return SP_EINVAL;
    if (layout != SP_ROTARY_HALF && layout != SP_ROTARY_INTERLEAVED) return SP_EINVAL;
    if (tokens < 0 || heads < 1 || heads > 65535 || width < 2 || width > 65536 || dim < 2 || dim % 2 || dim > width) return SP_ESHAPE;
    const uintptr_t low = dtype == SP_DTYPE_FP32 ? 3 : 1;
    if (!frequencies || ((uintptr_t)frequencies & 7) || (positions && cu_seqlens) || ((uintptr_t)positions & 3) || ((uintptr_t)cu_seqlens & 3))
        return SP_EINVAL;
    if (!positions && !cu_seqlens && tokens > 0) return SP_EINVAL;      // (positions of nothing may be null)
    if (cu_seqlens && batch < 0) return SP_ESHAPE;
    if (x_token < 0 || x_head < 0 || out_token < 0 || out_head < 0) return SP_ESHAPE;
    // (rows of the output that share memory would be written by several threads)
    if (!rows_apart(tokens, out_token, heads, out_head, width)) return SP_ESHAPE;
    if (x && x == out && (x_token != out_token || x_head != out_head)) return SP_EINVAL;
    // a thread per piece of a token: the grid holds 2^31 of them at most
    if ((int64_t)tokens * (width / 2 + 1) > INT32_MAX) return SP_ESHAPE;
    if (tokens == 0 || (cu_seqlens && batch == 0)) return SP_OK;
    if (!x || !out || ((uintptr_t)x & low) || ((uintptr_t)out & low)) return SP_EINVAL;
    return launch_rotary(x, x_token, x_head, out, out_token, out_head, dtype, tokens, heads, width, dim, layout, frequencies, factor,
                         positions, cu_seqlens, batch, 1, 0, 0, (hipStream_t)hip_stream) == hipSuccess ? SP_OK : SP_EHIP;
}

}  // extern "C"
