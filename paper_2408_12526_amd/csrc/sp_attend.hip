// Attention over packed sequences with capped scores, a bias by distance and masks (the definition is in sp_ops.h).
//
// One pass over the keys with the running maximum and sum of the softmax, products on the matrix cores.  The rows of a tile are (query, query
// head) pairs of one key head, r = query * share + head % share, so that heads that share keys share their tiles.  A wave takes 32 rows;
// per block of 32 keys:
//   S^T = K Q^T      (A operand: key rows from LDS; B operand: the rows' queries, in registers throughout)
//   scores           cap, slopes, table, mask: a row is a lane column, its keys sit in the registers of lanes l and l + 32; what a tile
//                    does not need (a mask where every row sees it all, the table where all distances are beyond its reach) is
//                    skipped by uniform branches
//   O^T += V^T P^T   (bf16: value fragments come transposed out of LDS by the transposing read; fp32: one value a lane)
// in two shapes: many rows, four waves with 32 rows each on the same key tiles; and few rows (up to 32 a sequence and key head, as one
// query against a long sequence), four waves with the same rows on key tiles of their own, joined at the end.  Either can be split over the
// keys where there are few workgroups; a small launch joins the parts.
//
// What bounds it: with many rows the vector instructions (a multiply-add, an exponential, a sum and half a maximum and conversion for a score: 28 cycles of
// a SIMD; a cap 24 to 44 more) and the products, 32 cycles each, which overlap only between the two (width 64: three) waves that the registers leave a
// SIMD.  bf16, 16 heads, 4 x 4096 tokens: width 128 on 4 key heads 660 us (830 TFLOP/s), causal 359, capped 786; width 64 361 (760), with slopes 429.
// With few rows the read of the keys and values: 8 queries of 32 heads on 4 key heads of 128 against 135 k keys, 270 MB, 65 us and 5 for the join (4.1
// TB/s without it).  Short sequences: the chain from the offsets to the first tile and out again, about 8 us a workgroup: 256 sequences of 57 tokens on
// average, 12 heads, 40 us.
#include <atomic>
#include <cfloat>
#include <cmath>

#include "sp_ops_internal.h"

namespace sp {

namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr int kWaveRows = 32;
enum { kMany, kSmall, kFew };          // shapes of a workgroup: 4 x 32 rows, 2 x 32 rows, 32 rows with the keys shared out to four waves
constexpr int kTablePad = 96;           // entries on each side of the table in LDS: a wave's 32 rows and a tile's 64 keys are less than that apart
constexpr int kRun = 16;                // neighbouring workgroups that stay on one XCD
constexpr int kTableBytes = 14336;      // largest table in LDS

// cap tanh(scale s / cap) in base-2 units, cap2 = cap log2(e), pre = 2 log2(e) scale / cap: tanh(y) = 1 - 2 / (e^(2 y) + 1), 2^-23 off in
// absolute value, far inside what bf16 operands leave of a score.
__device__ __forceinline__ float capped_far(float s, float pre, float cap2)
{
    return __builtin_fmaf(-2.f * cap2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s * pre) + 1.f), cap2);
}
// The same for |scale s / cap| < kNearCap, where five full-rate instructions do for two at a quarter of it and three more, and where
// fp32 needs it: tanh(y) = y (1 + y^2 (a + y^2 (b + y^2 c))), coefficients in terms of s
constexpr float kNearCap = 0.4f;
struct NearCap {
    float k0, k1, k2, k3;
};
__device__ __forceinline__ float capped_near(float s, const NearCap& k)
{
    const float t = s * s;
    return s * __builtin_fmaf(t, __builtin_fmaf(t, __builtin_fmaf(t, k.k3, k.k2), k.k1), k.k0);
}

struct AttendArgs {
    const char *q, *k, *v;
    char* out;
    float* lse;
    size_t qt, qh, kh, vh, ot, oh;                          // strides in bytes
    size_t qg, kg, vg, og;                                  // the same from group to group
    int kt, vt, slopes_g, bias_g, groups;                   // (slopes, bias: elements)
    const int32_t *cu_q, *cu_k, *prefix, *q_first, *doc_q, *doc_k;
    const float *slopes, *bias;
    float *part, *part_ml;                                  // [splits][total_q * heads][DP] sums, and (maximum, sum) pairs
    // Scores in base-2 units: raw ones (nothing but a positive scale) are multiplied where the exponential is taken.  cap2: the cap; pre: see
    // capped_far(); near_cap: |s| below which capped_near() does.
    float mult, pre, cap2, near_cap;
    NearCap cap_near;
    int from_start, raw, batch, heads, kv_heads, share, width, total_q, total_k, max_q, max_k, left, right, reach;
    int items, splits, table;                               // table: whether the bias is in LDS
};

// Sixteen bytes per lane from base + off, zeros from `bytes` on.  (All of the offset is the lane's: the hardware's check of the bound goes
// by that part.)
__device__ __forceinline__ u32x4 load16_bounded(const char* base, int bytes, unsigned off)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_raw_buffer_load_b128(__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, bytes, 0x00020000), (int)off, 0, 0);
#else
    return u32x4{};
#endif
}

__device__ __forceinline__ void sequence_range(int t0, int t1, int total, int most, int& at, int& n)
{
    at = t0 < 0 ? 0 : t0 > total ? total : t0;
    n = t1 - at;
    n = n < 0 ? 0 : n > most ? most : n;
    n = n > total - at ? total - at : n;
}

// A bias in units of the base-2 logarithm; finite ones stay finite, infinities and NaN what they are.
__device__ __forceinline__ float in_log2(float b) { return __builtin_isfinite(b) ? __builtin_amdgcn_fmed3f(b * kLog2e, -3.0e38f, 3.0e38f) : b; }

// From a row's reference (base-2 units) and sum: zero where it has seen nothing, else one at least, or NaN, which stays NaN.
__device__ __forceinline__ float lse_of(float top, float sum) { return sum == 0.f ? -INFINITY : (top + __builtin_log2f(sum)) * kLn2; }

template <class E, int DP, int KIND>
struct Shape {
    static constexpr bool B16 = sizeof(E) == 2, FEW = KIND == kFew;
    static constexpr int WAVES = KIND == kSmall ? 2 : 4, ROWS = FEW ? kWaveRows : WAVES * kWaveRows;
    static constexpr int KT = KIND == kMany && B16 ? 64 : 32;       // keys of a tile
    static constexpr int NT = FEW ? 64 : WAVES * 64;        // threads that fetch it
    static constexpr int RC = DP * (int)sizeof(E) / 16;     // 16-byte chunks of a row
    static constexpr int LPT = KT * RC / NT, RS = NT / RC;  // chunks a thread fetches, rows between them
    static constexpr int TILE = KT * RC * 16;               // bytes
    static constexpr int BUFS = FEW ? 4 : 2;                // FEW: one of each wave
    static constexpr int DOCS = BUFS * 2 * TILE, FOUND = DOCS + BUFS * KT * 4,
                         TABLE = FOUND + 128;                // offsets in LDS (FOUND: see the loop over tiles)
    static constexpr int JOIN = DOCS;                       // (FEW: maxima and sums of the waves, over the documents)
    static constexpr size_t LDS = FEW ? DOCS + 1024 : TABLE;
    static_assert(BUFS * 2 * TILE >= WAVES * kWaveRows * DP * (FEW ? 4 : (int)sizeof(E)), "the outputs reuse the tiles");
    // Chunk c of row r is in slot c ^ turn(r): the sixteen rows that a quarter of a read takes, or the four rows by four chunks of a
    // transposing one, lie in different banks.  Both turns are made of bits of r, so that of r + r' with no bit in common is the
    // exclusive or of theirs.
    static __host__ __device__ constexpr int key_turn(int r) { return RC == 8 ? (r >> 1) & 7 : r & 15; }
    static __host__ __device__ constexpr int value_turn(int r) { return !B16 ? (r >> 2 & 1) << 3 : RC == 8 ? (r >> 1 & 1) << 2 : (r & 3) << 2; }
    static __device__ __forceinline__ int key_slot(int r, int c) { return r * RC + (c ^ key_turn(r)); }
    static __device__ __forceinline__ int value_slot(int r, int c) { return r * RC + (c ^ value_turn(r)); }
};

// Waves on a SIMD that the registers are shared out for.
constexpr int waves_per_simd(bool b16, int dp, int kind, bool docs)
{
    return !b16 && dp == 128 ? (kind == kMany && !docs ? 2 : 1) : b16 && dp == 64 && kind != kFew && !(docs && kind == kMany) ? 3 : 2;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

template <class E, int DP, int KIND, bool DOCS>
__global__ __launch_bounds__((Shape<E, DP, KIND>::WAVES * 64), waves_per_simd(sizeof(E) == 2, DP, KIND, DOCS)) void attend_kernel(AttendArgs p)
{
    using S = Shape<E, DP, KIND>;
    constexpr bool FEW = S::FEW;
    constexpr int ROWS = S::ROWS, SHIFT = ROWS == 128 ? 7 : 6;
    constexpr int KT = S::KT, NB = KT / 32, RC = S::RC, LPT = S::LPT, RS = S::RS, ND = DP / 32;
    extern __shared__ char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j31 = lane & 31, g = lane >> 5;

    // ---- which rows ----
    int b, hk, m, r0, split, q0, nq, c0, c1;
    if (FEW) {
        b = blockIdx.x;
        m = blockIdx.y / p.kv_heads;
        hk = blockIdx.y - m * p.kv_heads;
        split = blockIdx.z;
        r0 = 0;
        c0 = p.cu_q[b];
        c1 = p.cu_q[b + 1];
    } else {
        // Neighbouring items of one key head read the same keys: runs of kRun stay on one XCD (workgroup id mod 8) and go round the XCDs,
        // another way each time, so that these have the same work whatever the lengths.  The last items come first: behind a causal
        // mask they are the longest, and what runs last should be short.
        const int total = p.items * p.kv_heads * p.splits * p.groups, y = (int)(gridDim.x >> 3) - 1 - (int)(blockIdx.x >> 3), round = y / kRun;
        const int lin = (round * 8 + (((int)blockIdx.x + round) & 7)) * kRun + y % kRun;
        if (lin >= total) return;
        split = lin % p.splits;
        const int item = lin / p.splits % p.items;
        hk = lin / p.splits / p.items;
        m = hk / p.kv_heads;
        hk -= m * p.kv_heads;
        // Item i belongs to the last sequence with cu * share / ROWS + b <= i: every sequence gets as many as it has blocks of rows, at least
        b = last_sequence(p.cu_q, p.batch, lane, [&](int i, int c) { return ((int64_t)c * p.share >> SHIFT) + i <= item; }, c0, c1);
        const int64_t start = (int64_t)item - (((int64_t)c0 * p.share >> SHIFT) + b);
        if (start < 0 || start > (1 << 23)) return;
        r0 = (int)start * ROWS;
    }
    sequence_range(c0, c1, p.total_q, p.max_q, q0, nq);
    const int rows = nq * p.share;
    if (r0 >= rows) return;                                 // (the whole workgroup)
    int k0, n;
    if (p.cu_k != p.cu_q) {                                 // (self-attention: the same offsets)
        c0 = p.cu_k[b];
        c1 = p.cu_k[b + 1];
    }
    sequence_range(c0, c1, p.total_k, p.max_k, k0, n);
    int first = p.q_first ? p.q_first[b] : p.from_start ? 0 : n - nq;
    first = first < -(1 << 30) ? -(1 << 30) : first > 1 << 30 ? 1 << 30 : first;
    int prefix = p.prefix ? p.prefix[b] : 0;
    prefix = prefix < 0 ? 0 : prefix > n ? n : prefix;

    const int rw = r0 + (FEW ? 0 : wave * kWaveRows);       // the wave's first row
    const bool idle = rw >= rows;
    const int r = rw + j31, rv = r < rows ? r : rows - 1, query = rv / p.share, head = hk * p.share + rv - query * p.share;
    const int pos = first + query;
    auto first_seen = [&](int i) { const int64_t x = p.left < 0 ? 0 : (int64_t)i - p.left; return (int)(x < 0 ? 0 : x > n ? n : x); };
    auto last_seen = [&](int i) { const int64_t x = p.right < 0 ? n - 1 : (int64_t)i + p.right; return (int)(x < -1 ? -1 : x > n - 1 ? n - 1 : x); };
    const int lo = first_seen(pos), hi = last_seen(pos);
    // of the wave: positions, and the keys that any and that every row sees
    const int rl = rw + kWaveRows - 1 < rows ? rw + kWaveRows - 1 : rows - 1;
    const int pos_a = first + (idle ? 0 : rw / p.share), pos_z = first + rl / p.share;
    const int any_lo = first_seen(pos_a), any_hi = last_seen(pos_z), all_lo = first_seen(pos_z), all_hi = last_seen(pos_a);

    // ---- which key tiles: those of the prefix, then those of the window of all the workgroup's rows ----
    const int re = r0 + ROWS - 1 < rows ? r0 + ROWS - 1 : rows - 1;
    const int w_lo = first_seen(first + r0 / p.share), w_hi = last_seen(first + re / p.share);
    const int tiles1 = (prefix + KT - 1) / KT, from2 = w_lo / KT > tiles1 ? w_lo / KT : tiles1, to2 = (w_hi + KT) / KT;     // (w_hi >= -1)
    const int tiles = tiles1 + (w_hi >= w_lo && to2 > from2 ? to2 - from2 : 0);
    const int per = (tiles + p.splits - 1) / p.splits, t_a = split * per, t_z = t_a + per < tiles ? t_a + per : tiles;
    auto tile_start = [&](int t) { return (t < tiles1 ? t : t - tiles1 + from2) * KT; };

    // ---- queries, table ----
    const char* qrow = p.q + m * p.qg + (size_t)(q0 + query) * p.qt + (size_t)head * p.qh;
    constexpr int QF = S::B16 ? DP / 16 : DP / 8;
    u32x4 qf[QF];                                           // bf16: dimensions 16 s + 8 g ..; fp32: 8 s + 4 g ..
#pragma unroll
    for (int s = 0; s < QF; ++s) {
        const int byte = (2 * s + g) * 16;
        qf[s] = byte < p.width * (int)sizeof(E) ? *(const u32x4*)(qrow + byte) : u32x4{0, 0, 0, 0};
    }
    const int doc = DOCS ? p.doc_q[q0 + query] : 0;
    const float slope = p.slopes ? p.slopes[m * p.slopes_g + head] * kLog2e : 0.f;
    float bias_left = 0.f, bias_right = 0.f;
    if (p.bias) {
        bias_left = in_log2(p.bias[(unsigned)(m * p.bias_g + head * (2 * p.reach + 1))]);
        bias_right = in_log2(p.bias[(unsigned)(m * p.bias_g + head * (2 * p.reach + 1) + 2 * p.reach)]);
    }
    float* table = (float*)(lds + S::TABLE);
    const int pitch = 2 * (p.reach + kTablePad) + 1;
    const float* tab = table + (head - hk * p.share) * pitch + p.reach + kTablePad;

    // ---- documents of the workgroup's rows ----
    int doc_lo = 0x7fffffff, doc_hi = -1;
    bool doc_one = true;                                    // all rows have the same one
    if (DOCS && !FEW) {
        for (int x = r0 / p.share + lane; x <= re / p.share; x += 64) {
            const int d = p.doc_q[q0 + x];
            if (d >= 0) {
                doc_lo = d < doc_lo ? d : doc_lo;
                doc_hi = d > doc_hi ? d : doc_hi;
            } else {
                doc_one = false;
            }
        }
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
            const int l = __shfl_xor(doc_lo, x), h = __shfl_xor(doc_hi, x);
            doc_lo = l < doc_lo ? l : doc_lo;
            doc_hi = h > doc_hi ? h : doc_hi;
        }
        doc_one = __all(doc_one) && doc_lo == doc_hi;
    }

    // ---- fetching: thread -> chunk fc of rows fr + i RS ----
    const int ft = FEW ? lane : tid, fc = ft % RC, fr = ft / RC;
    // Buffer loads from a tile's first row, bounded by the sequence's last row: what lies behind it, and chunks behind the width, come as
    // zeros.  One register of address per lane for each of the two.
    const bool inside = fc * 16 < p.width * (int)sizeof(E);
    const int k_at = inside ? fr * p.kt + fc * 16 : INT32_MAX, v_at = inside ? fr * p.vt + fc * 16 : INT32_MAX;
    const char* kbase = p.k + m * p.kg + (size_t)k0 * p.kt + (size_t)hk * p.kh;
    const char* vbase = p.v + m * p.vg + (size_t)k0 * p.vt + (size_t)hk * p.vh;
    u32x4 kr[LPT], vr[LPT];
    int dr[LPT], dk = 0;                                    // documents of the fetched rows; of the tile's key `ft` (FEW: lane i has row i's)
    auto fetch = [&](int j0, bool docs) {
        const int last = n - j0 < KT ? n - j0 - 1 : KT - 1;
        unsigned ka = (unsigned)k_at, va = (unsigned)v_at;  // (opaque: the rows' offsets are formed anew, kept they would spill)
        asm volatile("" : "+v"(ka), "+v"(va));
        const int kn = last * p.kt + p.width * (int)sizeof(E), vn = last * p.vt + p.width * (int)sizeof(E);
#pragma unroll
        for (int i = 0; i < LPT; ++i) {
            kr[i] = load16_bounded(kbase + (size_t)j0 * p.kt, kn, ka + (unsigned)(i * RS * p.kt));
            vr[i] = load16_bounded(vbase + (size_t)j0 * p.vt, vn, va + (unsigned)(i * RS * p.vt));
            if (DOCS && docs && !FEW) {
                const int j = j0 + fr + i * RS;
                dr[i] = p.doc_k[k0 + (j < n ? j : n - 1)];
            }
        }
        if (DOCS && docs && ft < KT) dk = p.doc_k[k0 + (j0 + ft < n ? j0 + ft : n - 1)];
    };
    const int key_to = S::key_slot(fr, fc) * 16, value_to = S::TILE + S::value_slot(fr, fc) * 16;
    char* const mine = lds + (FEW ? wave * 2 * S::TILE : 0);
    auto put = [&](int j0, int buf, bool docs) {
        char* to = mine + (FEW ? 0 : buf * 2 * S::TILE);
        if (DOCS && docs) {                                 // values that no row sees become zeros: a weight of zero does not hide a NaN
#pragma unroll
            for (int i = 0; i < LPT; ++i)
                if ((FEW ? __shfl(dk, fr + i * RS) : dr[i]) < 0) vr[i] = u32x4{0, 0, 0, 0};
        }
        int kto = key_to, vto = value_to;
        asm volatile("" : "+v"(kto), "+v"(vto));
#pragma unroll
        for (int i = 0; i < LPT; ++i) {
            constexpr int step = RS * RC * 16;
            *(u32x4*)(to + (kto ^ S::key_turn(i * RS) * 16) + i * step) = kr[i];
            *(u32x4*)(to + (vto ^ S::value_turn(i * RS) * 16) + i * step) = vr[i];
        }
        if (DOCS && docs && ft < KT) ((int*)(lds + S::DOCS))[(FEW ? wave : buf) * KT + ft] = dk;
    };

    // Short sequences: the first tile is requested before anything else is waited for.  (With documents it is not known yet.)
    const bool ahead = KIND == kSmall && !DOCS && t_a < t_z;
    if (ahead) fetch(tile_start(t_a), false);
    if (!FEW && p.table) {
        for (int h = 0; h < p.share; ++h)
            for (int e = tid; e < pitch; e += S::NT) {
                int d = e - kTablePad;
                d = d < 0 ? 0 : d > 2 * p.reach ? 2 * p.reach : d;
                table[h * pitch + e] = in_log2(p.bias[(unsigned)(m * p.bias_g + (hk * p.share + h) * (2 * p.reach + 1) + d)]);
            }
    }

    // ---- one tile ----
    f32x16 o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float mrun = -INFINITY, lrun = 0.f;                     // (of this half's keys)
    const bool raw = p.raw;
    const float mult = p.mult;
    // Where a lane reads key row j31, chunk g, and values: rows 4 g .. (bf16: a quarter wave's four rows by sixteen dimensions, eight bytes a
    // lane; fp32: dimension j31).  Rows further on are constants away: the swizzles go by bits of the row below those.
    const int key_at = S::key_slot(j31, g) * 16;
    const int value_at = S::TILE + (S::B16 ? S::value_slot(4 * g + ((lane & 15) >> 2), 2 * (lane >> 4 & 1) + ((lane & 3) >> 1)) * 16 + (lane & 1) * 8
                                           : S::value_slot(4 * g, j31 >> 2) * 16 + (j31 & 3) * 4);
    auto compute = [&](int j0, int buf, bool doc_mask) {
        const bool in_prefix = j0 < prefix;
        if (!in_prefix && (j0 > any_hi || j0 + KT <= any_lo)) return;       // (the wave sees none of it)
        // Addresses of the fragments are exclusive ors of two lane-dependent ones with constants (opaque here: kept in registers, all of
        // them together would spill).
        int kat = key_at, vat = value_at;
        asm volatile("" : "+v"(kat), "+v"(vat));
        const char* tile = mine + (FEW ? 0 : buf * 2 * S::TILE);
        f32x16 sc[NB];
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[nb][e] = 0.f;
#pragma unroll
            for (int s = 0; s < QF; ++s) {
                if (s % 4 == 0 && (s || nb)) __builtin_amdgcn_sched_barrier(0);     // (all fragments at once would not fit the registers)
                const u32x4 a = *(const u32x4*)(tile + (kat ^ (s * 32)) + nb * 32 * RC * 16);
                if constexpr (S::B16) {
                    sc[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, qf[s]), sc[nb], 0, 0, 0);
                } else {
                    const f32x4 fa = __builtin_bit_cast(f32x4, a), fq = __builtin_bit_cast(f32x4, qf[s]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[nb] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[e], fq[e], sc[nb], 0, 0, 0);
                }
            }
        }
        __builtin_amdgcn_s_setprio(0);
        // Register v of block nb is key j0 + 32 nb + 8 (v / 4) + 4 g + v % 4.
#define EACH_SCORE for (int nb = 0; nb < NB; ++nb) _Pragma("unroll") for (int v = 0; v < 16; ++v)
#define KEY_OFFSET (32 * nb + 8 * (v >> 2) + (v & 3))
        const int jg = j0 + 4 * g;
        if (!raw) {
            if (p.cap2 > 0.f) {
                if constexpr (S::B16) {
                    float far = 0.f;
#pragma unroll
                    EACH_SCORE far = __builtin_fmaxf(far, __builtin_fabsf(sc[nb][v]));
                    if (__all(far < p.near_cap)) {
#pragma unroll
                        EACH_SCORE sc[nb][v] = capped_near(sc[nb][v], p.cap_near);
                    } else {
#pragma unroll
                        EACH_SCORE sc[nb][v] = capped_far(sc[nb][v], p.pre, p.cap2);
                    }
                } else {
#pragma unroll
                    EACH_SCORE {
                        const float x = sc[nb][v], far = capped_far(x, p.pre, p.cap2);
                        sc[nb][v] = __builtin_fabsf(x) < p.near_cap ? capped_near(x, p.cap_near) : far;
                        if (v % 2) __builtin_amdgcn_sched_barrier(0);
                    }
                }
            } else {
#pragma unroll
                EACH_SCORE sc[nb][v] *= p.pre;
            }
            if (p.slopes) {
                const float d0 = (float)(jg - pos);
#pragma unroll
                EACH_SCORE sc[nb][v] = __builtin_fmaf(-slope, __builtin_fabsf(d0 + (float)KEY_OFFSET), sc[nb][v]);
            }
            if (p.bias) {
                if (j0 - pos_z >= p.reach) {
#pragma unroll
                    EACH_SCORE sc[nb][v] += bias_right;
                } else if (j0 + KT - 1 - pos_a <= -p.reach) {
#pragma unroll
                    EACH_SCORE sc[nb][v] += bias_left;
                } else if (!FEW && p.table) {
                    const float* at = tab + (jg - pos);
#pragma unroll
                    EACH_SCORE sc[nb][v] += at[KEY_OFFSET];
                } else {
                    // (32-bit offsets, few at a time: registers)
                    const unsigned at = (unsigned)(m * p.bias_g + head * (2 * p.reach + 1) + p.reach);
#pragma unroll
                    EACH_SCORE {
                        int d = jg + KEY_OFFSET - pos;
                        d = d < -p.reach ? -p.reach : d > p.reach ? p.reach : d;
                        sc[nb][v] += in_log2(p.bias[at + (unsigned)d]);
                        if (v % 2) __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        }
        if (!(j0 + KT <= prefix || (j0 >= all_lo && j0 + KT - 1 <= all_hi))) {
            const int a = lo - jg, z = hi - jg, pr = prefix - jg;
#pragma unroll
            EACH_SCORE if (!((KEY_OFFSET >= a && KEY_OFFSET <= z) || KEY_OFFSET < pr)) sc[nb][v] = -INFINITY;
        }
        if (DOCS && doc_mask) {
            const int* dt = (const int*)(lds + S::DOCS) + (FEW ? wave : buf) * KT + 4 * g;
#pragma unroll
            EACH_SCORE { const int x = dt[KEY_OFFSET]; if (x != doc || x < 0) sc[nb][v] = -INFINITY; }
        }
        float mx = sc[0][0];
#pragma unroll
        EACH_SCORE mx = __builtin_fmaxf(mx, sc[nb][v]);
        {
            float l = mx, h = mx;
            swap_halves(l, h);
            mx = __builtin_fmaxf(l, h);
        }
        // The reference of the exponentials is the maximum itself, so that the largest weight is one and bf16 does not round it.  (One that moves
        // where it is outgrown by 2^8 only: 642 us for 660, causal 345 for 359, width 64 351 for 361, in the shapes above; short sequences the same.)
        if (__any(mx > mrun)) {
            mx = __builtin_fmaxf(mx, mrun);
            const float alpha = mrun == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mrun - mx) * mult);
            mrun = mx;
            lrun *= alpha;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[d][e] *= alpha;
        }
        const float nm = mrun == -INFINITY ? 0.f : -mrun * mult;    // (a row that has seen nothing yet: weights 2^-inf)
        float psum = 0.f;
#pragma unroll
        EACH_SCORE {
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[nb][v], mult, nm));
            psum += e;
            sc[nb][v] = e;
        }
        lrun += psum;
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            if constexpr (S::B16) {
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2) {
                    bf16x8 pf;
#pragma unroll
                    for (int e = 0; e < 8; ++e) pf[e] = (bf16)sc[nb][8 * s2 + e];     // (half a step each: weights of 32 bits would take twice the products)
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        const char* at = tile + (vat ^ (d * 64)) + (32 * nb + 16 * s2) * RC * 16;
                        const s16x4 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
                        const s16x4 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 8 * RC * 16));
                        const bf16x8 va = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pf, o[d], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int v = 0; v < 16; ++v) {
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        const float va = *(const float*)(tile + (vat ^ (d * 128)) + (32 * nb + 8 * (v >> 2) + (v & 3)) * RC * 16);
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(va, sc[nb][v], o[d], 0, 0, 0);
                    }
                }
            }
        }
        __builtin_amdgcn_s_setprio(0);
#undef EACH_SCORE
#undef KEY_OFFSET
    };

    if (FEW) {
        constexpr bool docs = DOCS;
        for (int t = t_a + wave; t < t_z; t += 4) {
            if (t == t_a + wave) fetch(tile_start(t), docs);
            put(tile_start(t), 0, docs);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (t + 4 < t_z) fetch(tile_start(t + 4), docs);
            compute(tile_start(t), 0, docs);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    } else {
        int buf = 0;
        for (int base = t_a; base < t_z; base += 64) {
            const int m = t_z - base < 64 ? t_z - base : 64;
            unsigned long long live = m == 64 ? ~0ull : (1ull << m) - 1, masked = 0;
            if constexpr (DOCS) {
                // Four keys a lane, so that a load covers 256 of them; each wave looks at its share of the 64 tiles.  (Two places in LDS in turn:
                // a wave is at most one barrier ahead.)
                constexpr int LPK = KT / 4, TPL = 64 / LPK, OWN = 64 / S::WAVES;        // lanes of a tile, tiles of a load, tiles of a wave
                unsigned long long l = 0, u = 0;
#pragma unroll
                for (int i = 0; i < OWN; i += TPL) {
                    const int x0 = wave * OWN + i, t = x0 + lane / LPK, j = tile_start(base + (t < m ? t : m - 1)) + lane % LPK * 4;
                    bool any = false, all = doc_one;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int d = p.doc_k[k0 + (j + e < n ? j + e : n - 1)];
                        any = any || (d >= doc_lo && d <= doc_hi && j + e < n);
                        all = all && d == doc_lo && j + e < n;
                    }
                    // (bit 0 of every group of LPK lanes: whether any of the group says so)
                    unsigned long long some = __ballot(any), part = ~__ballot(all);
#pragma unroll
                    for (int x = LPK / 2; x; x >>= 1) {
                        some |= some >> x;
                        part |= part >> x;
                    }
#pragma unroll
                    for (int x = 0; x < TPL; ++x) {
                        l |= (some >> x * LPK & 1) << (x0 + x);
                        u |= (part >> x * LPK & 1) << (x0 + x);
                    }
                }
                unsigned long long* found = (unsigned long long*)(lds + S::FOUND) + (base - t_a >> 6 & 1) * 8;
                if (lane == 0) {
                    found[wave] = l;
                    found[4 + wave] = u;
                }
                barrier_lds();
                l = 0;
#pragma unroll
                for (int w = 0; w < S::WAVES; ++w) {
                    l |= found[w];
                    masked |= found[4 + w];
                }
                live &= ((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(l >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)l);
                masked = ((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(masked >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)masked);
            }
            if (!live) continue;
            int t = __builtin_ctzll(live);
            if (!ahead || base > t_a) fetch(tile_start(base + t), masked >> t & 1);
            for (;;) {
                const int j0 = tile_start(base + t);
                const bool doc_mask = masked >> t & 1;
                put(j0, buf, doc_mask);
                live &= live - 1;
                barrier_lds();
                if (live) {
                    t = __builtin_ctzll(live);
                    fetch(tile_start(base + t), masked >> t & 1);
                }
                if (!idle) compute(j0, buf, doc_mask);
                buf ^= 1;
                if (!live) break;
            }
        }
    }

    // ---- results ----
    {
        float l = lrun, h = lrun;
        swap_halves(l, h);
        lrun = l + h;
    }
    float m2 = mrun == -INFINITY ? -INFINITY : mrun * mult;     // base-2 units
    if (FEW) {
        // The waves' sums, 32 rows x DP each in the wave's own tile (chunk c of row r in slot c ^ (r % 16)), maxima and sums behind
        float* ml = (float*)(lds + S::JOIN);
        barrier_lds();                                      // (documents are read no more)
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4) {
                const int c = 8 * d + 2 * v4 + g;
                *(f32x4*)(mine + (j31 * (DP / 4) + (c ^ (j31 & 15))) * 16) = f32x4{o[d][4 * v4], o[d][4 * v4 + 1], o[d][4 * v4 + 2], o[d][4 * v4 + 3]};
            }
        if (g == 0) {
            ml[(wave * 32 + j31) * 2] = m2;
            ml[(wave * 32 + j31) * 2 + 1] = lrun;
        }
        barrier_lds();
        constexpr int TPR = 8, CPT = DP / 4 / TPR;          // threads of a row, chunks of four of each
        const int row = tid / TPR, cc = tid % TPR;
        if (row >= rows) return;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = __builtin_fmaxf(top, ml[(w * 32 + row) * 2]);
        float f[4], sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float m = ml[(w * 32 + row) * 2];
            f[w] = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
            sum += f[w] * ml[(w * 32 + row) * 2 + 1];
        }
        const int qu = row / p.share, he = hk * p.share + row - qu * p.share;
        const size_t at = ((size_t)m * p.total_q + q0 + qu) * p.heads + he;
        const float inv = p.splits > 1 ? 1.f : sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const int c = cc + TPR * i;
            if (c * 4 >= p.width) continue;
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const f32x4 y = *(const f32x4*)(lds + w * 2 * S::TILE + (row * (DP / 4) + (c ^ (row & 15))) * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] += f[w] * y[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] *= inv;
            if (p.splits > 1) {
                *(f32x4*)(p.part + ((size_t)split * p.groups * p.total_q * p.heads + at) * DP + c * 4) = x;
            } else {
                E* out = (E*)(p.out + m * p.og + (size_t)(q0 + qu) * p.ot + (size_t)he * p.oh) + c * 4;
                if constexpr (S::B16) *(bf16x4*)out = bf16x4{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
                else *(f32x4*)out = x;
            }
        }
        if (cc == 0) {
            if (p.splits > 1) {
                float* to = p.part_ml + ((size_t)split * p.groups * p.total_q * p.heads + at) * 2;
                to[0] = top;
                to[1] = sum;
            } else if (p.lse) {
                p.lse[at] = lse_of(top, sum);
            }
        }
        return;
    }
    const size_t at = ((size_t)m * p.total_q + q0 + query) * p.heads + head;
    if (p.splits > 1) {
        if (r >= rows) return;
        const size_t row = (size_t)split * p.groups * p.total_q * p.heads + at;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4)
                *(f32x4*)(p.part + row * DP + 32 * d + 8 * v4 + 4 * g) = f32x4{o[d][4 * v4], o[d][4 * v4 + 1], o[d][4 * v4 + 2], o[d][4 * v4 + 3]};
        if (g == 0) {
            p.part_ml[row * 2] = m2;
            p.part_ml[row * 2 + 1] = lrun;
        }
        return;
    }
    if (g == 0 && r < rows && p.lse) p.lse[at] = lse_of(m2, lrun);
    barrier_lds();                                          // (the tiles are read no more)
    if (idle) return;
    // The wave's 32 rows leave through its quarter of the tiles as whole rows.
    const float inv = lrun > 0.f ? 1.f / lrun : 0.f;
    char* stage = lds + wave * kWaveRows * RC * 16;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4) {
            const int byte = (32 * d + 8 * v4 + 4 * g) * (int)sizeof(E), c = byte >> 4;
            char* to = stage + (j31 * RC + (c ^ (RC == 8 ? j31 & 7 : j31 & 15))) * 16 + (byte & 15);
            if constexpr (S::B16)
                *(bf16x4*)to = bf16x4{(bf16)(o[d][4 * v4] * inv), (bf16)(o[d][4 * v4 + 1] * inv), (bf16)(o[d][4 * v4 + 2] * inv), (bf16)(o[d][4 * v4 + 3] * inv)};
            else
                *(f32x4*)to = f32x4{o[d][4 * v4] * inv, o[d][4 * v4 + 1] * inv, o[d][4 * v4 + 2] * inv, o[d][4 * v4 + 3] * inv};
        }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    constexpr int RPI = 64 / RC;                            // rows an instruction stores
    const int oc = lane % RC;
    if (oc * 16 < p.width * (int)sizeof(E))
#pragma unroll
        for (int x = 0; x < kWaveRows; x += RPI) {
            const int row = x + lane / RC, rr = rw + row;
            if (rr >= rows) break;
            const int qu = rr / p.share, he = hk * p.share + rr - qu * p.share;
            *(u32x4*)(p.out + m * p.og + (size_t)(q0 + qu) * p.ot + (size_t)he * p.oh + oc * 16) = *(const u32x4*)(stage + (row * RC + (oc ^ (RC == 8 ? row & 7 : row & 15))) * 16);
        }
}

// A wave joins the parts of one query and head.
template <class E, int DP>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs p)
{
    const int lane = threadIdx.x & 63, b = blockIdx.z % p.batch, m = blockIdx.z / p.batch, head = blockIdx.y, r = blockIdx.x * 4 + (threadIdx.x >> 6);
    int q0, nq;
    sequence_range(p.cu_q[b], p.cu_q[b + 1], p.total_q, p.max_q, q0, nq);
    if (r >= nq) return;
    const size_t step = (size_t)p.groups * p.total_q * p.heads, at = ((size_t)m * p.total_q + q0 + r) * p.heads + head;
    float top = -INFINITY;
    for (int s = lane; s < p.splits; s += 64) top = __builtin_fmaxf(top, p.part_ml[(s * step + at) * 2]);
    top = wave_max(top);
    float sum = 0.f, x0 = 0.f, x1 = 0.f;
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) {
        const float m = p.part_ml[(s * step + at) * 2], f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        sum += f * p.part_ml[(s * step + at) * 2 + 1];
        const float* x = p.part + (s * step + at) * DP;
        x0 += f * x[lane];
        if (DP > 64) x1 += f * x[lane + 64];
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    E* out = (E*)(p.out + m * p.og + (size_t)(q0 + r) * p.ot + (size_t)head * p.oh);
    if (lane < p.width) out[lane] = (E)(x0 * inv);
    if (DP > 64 && lane + 64 < p.width) out[lane + 64] = (E)(x1 * inv);
    if (p.lse && lane == 0) p.lse[at] = lse_of(top, sum);
}

struct Plan {
    int kind, dp, items, splits;
    size_t part, ml;                    // bytes
};

// Shape of the workgroups: few rows where no sequence has more than 32, small where they have up to 96 (fp32, whose waves the matrix
// products keep busy for longer: 192) on average, of 128 rows half the waves being idle then.  us a call in a graph, small / many, width 64:
// fp32, 8 heads, 32 sequences of 158 on average 48 / 64, of 128 25 / 25, 192 37 / 47, 224 67 / 54, 2 of 2048 277 / 217; bf16, 16 heads, 64 sequences of 64
// 13.7 / 13.3, 80 16.8 / 18.2, 96 16.1 / 18.6, 112 19.9 / 19.7, 128 20.2 / 24.2, 192 35 / 31, 256 43 / 40, 4 of 4096 437 / 362; 12 heads, 256 sequences of 57 on
// average 33 / 41.  Parts of a call: as many as give every compute unit two workgroups, of at least 256 keys for each wave (few
// rows) or 512 for all of them.
Plan make_plan(const sp_attention_args& a, int groups, bool split)
{
    Plan P{};
    const int share = a.heads / a.kv_heads;
    P.kind = (int64_t)a.max_q * share <= kWaveRows ? kFew : (int64_t)a.total_q * share <= (int64_t)(a.dtype == SP_DTYPE_FP32 ? 192 : 96) * a.batch ? kSmall : kMany;
    P.dp = a.width <= 64 ? 64 : 128;
    const int rows = P.kind == kMany ? 128 : 64;
    P.items = P.kind == kFew ? a.batch : (int)((int64_t)a.total_q * share / rows) + a.batch;
    const int64_t blocks = (P.kind == kFew ? (int64_t)a.batch : ((int64_t)a.max_q * share + rows - 1) / rows * a.batch) * a.kv_heads * groups;
    const int64_t want = (512 + blocks - 1) / blocks, most = a.max_k / (P.kind == kFew ? 1024 : 512);
    P.splits = (int)(want < most ? want : most);
    P.splits = P.splits < 1 || !split ? 1 : P.splits > 64 ? 64 : P.splits;
    if (P.splits > 1) {
        const size_t rows = (size_t)P.splits * groups * a.total_q * a.heads;
        P.part = rows * P.dp * 4;
        P.ml = rows * 8;
    }
    return P;
}

template <class E, int DP, int KIND, bool DOCS>
hipError_t launch_shape(const AttendArgs& a, const Plan& P, hipStream_t s)
{
    using S = Shape<E, DP, KIND>;
    const size_t smem = S::LDS + (!S::FEW && a.table ? (size_t)a.share * (2 * (a.reach + kTablePad) + 1) * 4 : 0);
    auto kern = attend_kernel<E, DP, KIND, DOCS>;
    static std::atomic<size_t> raised{0};                   // per instantiation; the attribute is sticky for the process
    if (smem > 48 * 1024 && raised.load(std::memory_order_acquire) < smem) {
        const size_t most = S::LDS + (S::FEW ? 0 : kTableBytes);
        const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)most);
        if (e != hipSuccess) return e;
        raised.store(most, std::memory_order_release);
    }
    const dim3 grid = S::FEW ? dim3((unsigned)a.batch, (unsigned)(a.kv_heads * a.groups), (unsigned)P.splits)
                          : dim3((unsigned)(((int64_t)P.items * a.kv_heads * P.splits * a.groups + 8 * kRun - 1) / (8 * kRun) * (8 * kRun)));
    hipLaunchKernelGGL(kern, grid, dim3(S::WAVES * 64), smem, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || P.splits == 1) return e;
    hipLaunchKernelGGL((attend_join_kernel<E, DP>), dim3((unsigned)((a.max_q + 3) / 4), (unsigned)a.heads, (unsigned)(a.batch * a.groups)), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <class E, int DP, int KIND>
hipError_t launch_docs(const AttendArgs& a, const Plan& P, hipStream_t s)
{
    return a.doc_k ? launch_shape<E, DP, KIND, true>(a, P, s) : launch_shape<E, DP, KIND, false>(a, P, s);
}

template <class E, int DP>
hipError_t launch_kind(const AttendArgs& a, const Plan& P, hipStream_t s)
{
    return P.kind == kFew ? launch_docs<E, DP, kFew>(a, P, s) : P.kind == kSmall ? launch_docs<E, DP, kSmall>(a, P, s) : launch_docs<E, DP, kMany>(a, P, s);
}

template <class E>
hipError_t launch_type(const AttendArgs& a, const Plan& P, hipStream_t s)
{
    return P.dp == 64 ? launch_kind<E, 64>(a, P, s) : launch_kind<E, 128>(a, P, s);
}

}  // namespace

size_t attend_workspace_bytes(const sp_attention_args& a)
{
    const Plan P = make_plan(a, 1, true);
    return P.part + P.ml;
}

hipError_t launch_attend(const sp_attention_args& a, const AttendGroups& g, void* workspace, hipStream_t s)
{
    const Plan P = make_plan(a, g.groups, workspace != nullptr);
    const size_t sz = a.dtype == SP_DTYPE_FP32 ? 4 : 2;
    AttendArgs d{};
    d.q = (const char*)a.q; d.k = (const char*)a.k; d.v = (const char*)a.v; d.out = (char*)a.out; d.lse = a.lse;
    d.qt = a.q_token * sz; d.qh = a.q_head * sz; d.kt = (int)(a.k_token * sz); d.kh = a.k_head * sz;
    d.vt = (int)(a.v_token * sz); d.vh = a.v_head * sz; d.ot = a.out_token * sz; d.oh = a.out_head * sz;
    d.cu_q = a.cu_q; d.cu_k = a.cu_k; d.prefix = a.prefix; d.q_first = a.q_first; d.doc_q = a.doc_q; d.doc_k = a.doc_k;
    d.slopes = a.slopes; d.bias = a.bias;
    d.part = (float*)workspace; d.part_ml = (float*)((char*)workspace + P.part);
    const float ratio = a.cap > 0.f ? a.scale / a.cap : 0.f, k0 = a.scale * kLog2e, r2 = ratio * ratio;
    d.raw = !(a.cap > 0.f) && !a.slopes && !a.bias && a.scale > 0.f;
    d.mult = d.raw ? k0 : 1.f;
    d.cap2 = a.cap > 0.f ? a.cap * kLog2e : 0.f;
    // (finite for the smallest cap as well: zero scores are multiplied by it)
    d.pre = a.cap > 0.f ? std::fmin(std::fmax(ratio * (2.f * kLog2e), -FLT_MAX), FLT_MAX) : k0;
    d.near_cap = kNearCap / std::fabs(ratio);
    // (the least-squares fit of tanh(y) on |y| < 0.4, reweighted until its errors were even: 2.8e-8)
    d.cap_near = NearCap{k0, -0.33331388f * k0 * r2, 0.13268751f * k0 * r2 * r2, -0.04742304f * k0 * r2 * r2 * r2};
    // A cap so small that the coefficients leave fp32: capped_far() alone, whose 2^-23 of that cap is nothing
    if (!std::isfinite(d.cap_near.k3)) {
        d.near_cap = 0.f;
        d.cap_near = NearCap{};
    }
    d.batch = a.batch; d.heads = a.heads; d.kv_heads = a.kv_heads; d.share = a.heads / a.kv_heads; d.width = a.width;
    d.total_q = a.total_q; d.total_k = a.total_k; d.max_q = a.max_q; d.max_k = a.max_k; d.left = a.left; d.right = a.right; d.reach = a.reach;
    d.qg = g.q * sz; d.kg = g.k * sz; d.vg = g.v * sz; d.og = g.out * sz; d.slopes_g = a.slopes ? (int)g.slopes : 0; d.bias_g = a.bias ? (int)g.bias : 0;
    d.groups = g.groups; d.from_start = g.from_start; d.items = P.items; d.splits = P.splits;
    d.table = a.bias && (int64_t)d.share * (2 * ((int64_t)a.reach + kTablePad) + 1) * 4 <= kTableBytes;
    return a.dtype == SP_DTYPE_FP32 ? launch_type<float>(d, P, s) : launch_type<bf16>(d, P, s);
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
    constexpr int32_t most = 1 << 29;                      // (positions and distances stay inside 32 bits)
    if (a->batch > 65535 || a->total_q > most || a->total_k > most || a->total_q < 0 || a->total_k < 0 || a->max_q < 0 || a->max_k < 0) return SP_ESHAPE;
    if ((int64_t)a->total_q * a->heads > (1 << 30) || (int64_t)a->batch * a->heads > (1 << 22)) return SP_ESHAPE;
    if (!std::isfinite(a->scale) || !std::isfinite(a->cap) || a->reach < 0 || a->reach > (1 << 20)) return SP_EINVAL;
    if (a->bias && (int64_t)a->heads * (2 * (int64_t)a->reach + 1) > (1 << 30)) return SP_ESHAPE;
    // (one of nothing may be null)
    if ((a->doc_q && !a->doc_k && a->total_k > 0) || (a->doc_k && !a->doc_q && a->total_q > 0)) return SP_EINVAL;
    const int sz = a->dtype == SP_DTYPE_FP32 ? 4 : 2;
    const int64_t strides[] = {a->q_token, a->q_head, a->k_token, a->k_head, a->v_token, a->v_head, a->out_token, a->out_head};
    for (int64_t s : strides) {
        if (s < 0 || s > most) return SP_ESHAPE;
        if (s * sz & 15) return SP_EINVAL;
    }
    if (a->k_token > (1 << 23) || a->v_token > (1 << 23)) return SP_ESHAPE;         // (offsets inside a tile of 64 rows are 32-bit)
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
    return launch_attend(*args, AttendGroups{1, 0, 0, 0, 0, 0, 0, false}, need ? workspace : nullptr, (hipStream_t)hip_stream) == hipSuccess ? SP_OK : SP_EHIP;
}

}  // extern "C"
