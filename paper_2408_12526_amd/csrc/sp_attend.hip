// Attention over packed sequences with capped scores, a bias by distance and masks (the definition is in sp_ops.h).
#include <cmath>

#include "sp_ops_internal.h"

namespace sp {

namespace {

// A wave takes one query of one head: a lane a key for the scores, a lane two dimensions for the values.
template <class E>
__global__ __launch_bounds__(256) void attend_simple_kernel(sp_attention_args p)
{
    const int lane = threadIdx.x & 63, h = blockIdx.y, b = blockIdx.z;
    const int r = blockIdx.x * 4 + (threadIdx.x >> 6);
    auto range = [](const int32_t* cu, int b, int total, int most, int& t0, int& n) {
        t0 = cu[b];
        t0 = t0 < 0 ? 0 : t0 > total ? total : t0;
        n = cu[b + 1] - t0;
        n = n < 0 ? 0 : n > most ? most : n;
        n = n > total - t0 ? total - t0 : n;
    };
    int q0, nq, k0, nk;
    range(p.cu_q, b, p.total_q, p.max_q, q0, nq);
    range(p.cu_k, b, p.total_k, p.max_k, k0, nk);
    if (r >= nq) return;
    const int i = (p.q_first ? p.q_first[b] : nk - nq) + r, t = q0 + r, hk = h / (p.heads / p.kv_heads);
    const E* q = (const E*)p.q + t * p.q_token + h * p.q_head;
    const int doc = p.doc_q ? p.doc_q[t] : 0, prefix = p.prefix ? p.prefix[b] : 0;
    float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
    for (int j0 = 0; j0 < nk; j0 += 64) {
        const int j = j0 + lane, d = j - i;
        bool seen = j < nk && (((p.left < 0 || d >= -p.left) && (p.right < 0 || d <= p.right)) || j < prefix);
        if (seen && p.doc_k) { const int dk = p.doc_k[k0 + j]; seen = dk == doc && dk >= 0; }
        float s = -INFINITY;
        if (seen) {
            const E* k = (const E*)p.k + (k0 + j) * p.k_token + hk * p.k_head;
            s = 0.f;
            for (int e = 0; e < p.width; ++e) s = __builtin_fmaf((float)q[e], (float)k[e], s);
            s *= p.scale;
            if (p.cap > 0.f) s = p.cap * tanhf(s / p.cap);
            if (p.slopes) s -= p.slopes[h] * fabsf((float)d);
            if (p.bias) s += p.bias[(size_t)h * (2 * p.reach + 1) + (d < -p.reach ? -p.reach : d > p.reach ? p.reach : d) + p.reach];
        }
        const float mn = fmaxf(m, wave_max(s));
        if (mn == -INFINITY) continue;
        const float al = expf(m - mn), e = expf(s - mn);
        l = l * al + wave_sum(e);
        o0 *= al;
        o1 *= al;
        m = mn;
        for (int c = 0; c < 64 && j0 + c < nk; ++c) {
            const float w = __shfl(e, c);
            if (w == 0.f) continue;
            const E* v = (const E*)p.v + (k0 + j0 + c) * p.v_token + hk * p.v_head;
            if (lane < p.width) o0 += w * (float)v[lane];
            if (lane + 64 < p.width) o1 += w * (float)v[lane + 64];
        }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    E* out = (E*)p.out + t * p.out_token + h * p.out_head;
    if (lane < p.width) out[lane] = (E)(o0 * inv);
    if (lane + 64 < p.width) out[lane + 64] = (E)(o1 * inv);
    if (p.lse && lane == 0) p.lse[(size_t)t * p.heads + h] = l > 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace

size_t attend_workspace_bytes(const sp_attention_args&) { return 0; }

hipError_t launch_attend(const sp_attention_args& a, void*, hipStream_t s)
{
    const dim3 grid((unsigned)((a.max_q + 3) / 4), (unsigned)a.heads, (unsigned)a.batch);
    if (a.dtype == SP_DTYPE_FP32) hipLaunchKernelGGL(attend_simple_kernel<float>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(attend_simple_kernel<bf16>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace sp

using namespace sp;

namespace {

// What is wrong with the arguments but for the workspace; SP_OK: nothing.
int check_attention(const sp_attention_args* a)
{
    if (!a) return SP_EINVAL;
    if (a->dtype != SP_DTYPE_FP32 && a->dtype != SP_DTYPE_BF16) return SP_EINVAL;
    if (a->batch < 0 || a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads || a->heads > 65535) return SP_ESHAPE;
    if (a->width < 8 || a->width > 128 || a->width % 8) return SP_ESHAPE;
    if (a->batch > 65535 || a->total_q < 0 || a->total_k < 0 || a->max_q < 0 || a->max_k < 0) return SP_ESHAPE;
    if (!std::isfinite(a->scale) || !std::isfinite(a->cap) || a->reach < 0 || a->reach > (1 << 20)) return SP_EINVAL;
    if (!a->doc_q != !a->doc_k) return SP_EINVAL;
    const int sz = a->dtype == SP_DTYPE_FP32 ? 4 : 2;
    const int64_t strides[] = {a->q_token, a->q_head, a->k_token, a->k_head, a->v_token, a->v_head, a->out_token, a->out_head};
    for (int64_t s : strides) {
        if (s < 0) return SP_ESHAPE;
        if (s * sz & 15) return SP_EINVAL;
    }
    if (!rows_apart(a->total_q, a->out_token, a->heads, a->out_head, a->width)) return SP_ESHAPE;
    const void* rows[] = {a->q, a->k, a->v, a->out};
    for (const void* p : rows)
        if ((uintptr_t)p & 15) return SP_EINVAL;
    const void* words[] = {a->lse, a->cu_q, a->cu_k, a->prefix, a->q_first, a->doc_q, a->doc_k, a->slopes, a->bias};
    for (const void* p : words)
        if ((uintptr_t)p & 3) return SP_EINVAL;
    if (a->total_q > 0 && (!a->q || !a->out || !a->cu_q || !a->cu_k || (a->total_k > 0 && (!a->k || !a->v)))) return SP_EINVAL;
    if (a->total_q > 0 && (a->out == a->q || a->out == a->k || a->out == a->v)) return SP_EINVAL;
    return SP_OK;
}

}  // namespace

extern "C" {

size_t sp_attention_workspace_bytes(const sp_attention_args* args)
{
    return check_attention(args) == SP_OK && args->total_q > 0 && args->batch > 0 && args->max_q > 0 ? attend_workspace_bytes(*args) : 0;
}

int sp_attention(const sp_attention_args* args, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const int rc = check_attention(args);
    if (rc != SP_OK) return rc;
    if (args->total_q == 0 || args->batch == 0 || args->max_q == 0) return SP_OK;
    const size_t need = attend_workspace_bytes(*args);
    if (need && (!workspace || ((uintptr_t)workspace & 255))) return SP_EINVAL;
    if (workspace_bytes < need) return SP_ENOMEM;
    return launch_attend(*args, workspace, (hipStream_t)hip_stream) == hipSuccess ? SP_OK : SP_EHIP;
}

}  // extern "C"
