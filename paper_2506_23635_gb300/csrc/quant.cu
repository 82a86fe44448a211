// 8-bit experts: quantisation in blocks of 128, the choice of experts from logits, and
// the C ABI of the grouped products and of the layer over them (include/moe.h).
#include <math.h>

#include "layer_steps.cuh"
#include "quant.cuh"

namespace moe {
namespace {

// ===========================================================================
// Quantising rows: 16 lanes take a block of 128 numbers, eight each.  Bound by memory
// (8190 x 6144 bf16: 27.5 us, 5.6 TB/s read and written, 0.82 of a copy's rate).
// With K > 0 the rows are tokens, each written to the K sorted positions of its
// slots (inv_perm; -1: left out), so that a token is read and quantised once, and
// the scales block by block ([blocks, rows * K]), as the products read them.
// ===========================================================================
constexpr int kRowsThreads = 256;

template <typename TX, int U>
__global__ void __launch_bounds__(kRowsThreads)
k_quant_rows(int rows, int cols, int K, const TX *__restrict__ x,
             const int32_t *__restrict__ inv_perm, uint8_t *__restrict__ q,
             float *__restrict__ scale, int *__restrict__ count, int n_count) {
    ptx::grid_dependency_wait();
    ptx::launch_dependents();  // (after the wait: the products read offsets and weights early)
    if (count && blockIdx.x == 0)
        for (int i = threadIdx.x; i < n_count; i += kRowsThreads) count[i] = 0;
    const int nb = q_blocks(cols), sub = threadIdx.x & 15;
    // blocks of a row in runs of U; 16 lanes take a run (the shuffles take whole warps, so
    // both halves of a warp go on to its last run)
    const unsigned runs = (unsigned)(nb + U - 1) / U;
    const long long items = (long long)rows * runs, stride = (long long)gridDim.x * (kRowsThreads / 16);
    const long long first = (long long)blockIdx.x * (kRowsThreads / 16) + (threadIdx.x >> 4);
    for (long long i = first; i - (threadIdx.x >> 4 & 1) < items; i += stride) {
        const bool in = i < items;
        const int row = in ? (int)(i / runs) : 0, b0 = in ? (int)(i - (long long)row * runs) * U : nb;
        const TX *src = x + (size_t)row * cols + sub * 8;
        float v[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if ((b0 + u) * 128 + sub * 8 < cols) stream8(src + (b0 + u) * 128, v[u]);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) v[u][j] = 0.f;
        }
        float sc[U];
        uint2 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v[u][j]));
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
            float inv;
            q_scale(m, sc[u], inv);
            w[u] = make_uint2(q_pack4(v[u][0], v[u][1], v[u][2], v[u][3], inv),
                              q_pack4(v[u][4], v[u][5], v[u][6], v[u][7], inv));
        }
        const int copies = K > 0 ? K : 1;
        for (int k = 0; in && k < copies; ++k) {
            const int j = K > 0 ? inv_perm[(size_t)row * K + k] : row;
            if (j < 0) continue;
            uint8_t *to = q + (size_t)j * cols + sub * 8;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int b = b0 + u;
                if (b * 128 + sub * 8 < cols) *reinterpret_cast<uint2 *>(to + b * 128) = w[u];
                if (sub == u && b < nb)
                    scale[K > 0 ? (size_t)b * rows * K + j : (size_t)j * nb + b] = sc[u];
            }
        }
    }
}

// Quantising matrices: a block of 256 threads holds 128 x 128 numbers in registers, as
// they were loaded.  Bound by memory (four of 10752 x 6144 bf16: 121 us, 0.97 of a copy's rate).
__device__ __forceinline__ void hold8(const bf16 *p, uint4 (&r)[1]) { r[0] = ld_stream16(p); }
__device__ __forceinline__ void hold8(const float *p, uint4 (&r)[2]) {
    r[0] = ld_stream16(p);
    r[1] = ld_stream16(p + 4);
}
__device__ __forceinline__ void held8(const uint4 (&r)[1], float (&o)[8]) {
    unpack_bf16x2(r[0].x, o[0], o[1]);
    unpack_bf16x2(r[0].y, o[2], o[3]);
    unpack_bf16x2(r[0].z, o[4], o[5]);
    unpack_bf16x2(r[0].w, o[6], o[7]);
}
__device__ __forceinline__ void held8(const uint4 (&r)[2], float (&o)[8]) {
    o[0] = __uint_as_float(r[0].x); o[1] = __uint_as_float(r[0].y);
    o[2] = __uint_as_float(r[0].z); o[3] = __uint_as_float(r[0].w);
    o[4] = __uint_as_float(r[1].x); o[5] = __uint_as_float(r[1].y);
    o[6] = __uint_as_float(r[1].z); o[7] = __uint_as_float(r[1].w);
}

template <typename TX>
__global__ void __launch_bounds__(256)
k_quant_blocks(int rows, int cols, const TX *__restrict__ w, uint8_t *__restrict__ q,
               float *__restrict__ scale) {
    __shared__ uint32_t red[8];
    const int nb = q_blocks(cols), nr = q_blocks(rows);
    const unsigned blk = blockIdx.x;
    const int b = (int)(blk % nb), r = (int)(blk / nb % nr);
    const unsigned n = blk / nb / nr;
    const int c = b * 128 + (threadIdx.x & 15) * 8, r0 = r * 128 + (threadIdx.x >> 4);
    const size_t base = (size_t)n * rows * cols + c;
    uint4 v[8][sizeof(TX) / 2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = r0 + 16 * i;
        if (row < rows && c < cols) hold8(w + base + (size_t)row * cols, v[i]);
        else
#pragma unroll
            for (int j = 0; j < (int)sizeof(TX) / 2; ++j) v[i][j] = make_uint4(0, 0, 0, 0);
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float f[8];
        held8(v[i], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, abs_bits(f[j]));
    }
    m = __reduce_max_sync(0xffffffffu, m);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, red[i]);
    float sc, inv;
    q_scale(m, sc, inv);
    if (threadIdx.x == 0) scale[blk] = sc;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = r0 + 16 * i;
        if (row < rows && c < cols) {
            float f[8];
            held8(v[i], f);
            *reinterpret_cast<uint2 *>(q + base + (size_t)row * cols) =
                make_uint2(q_pack4(f[0], f[1], f[2], f[3], inv), q_pack4(f[4], f[5], f[6], f[7], inv));
        }
    }
}

// Ahead of a product: its rows' scales [S, nb] block by block, counters of zero.
__global__ void __launch_bounds__(256)
k_quant_scales(int S, int nb, const float *__restrict__ in, float *__restrict__ out, int *count,
               int n_count) {
    __shared__ float tile[32][33];
    ptx::grid_dependency_wait();
    ptx::launch_dependents();  // (after the wait: the product reads offsets and weights early)
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = threadIdx.x; i < n_count; i += 256) count[i] = 0;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, b0 = blockIdx.y * 32;
    for (int s0 = blockIdx.x * 32; s0 < S; s0 += gridDim.x * 32) {
#pragma unroll
        for (int i = y; i < 32; i += 8)
            if (s0 + i < S && b0 + x < nb) tile[i][x] = in[(size_t)(s0 + i) * nb + b0 + x];
        __syncthreads();
#pragma unroll
        for (int i = y; i < 32; i += 8)
            if (b0 + i < nb && s0 + x < S) out[(size_t)(b0 + i) * S + s0 + x] = tile[x][i];
        __syncthreads();
    }
}

// ===========================================================================
// The choice of experts: one warp a token, lane i the experts [i NE, (i + 1) NE).  Scores
// and keys in 32 bits first; where two of the keys that decide lie nearer to each other
// than the error of 32 bits, the warp does the token again with more, so that the choice
// is that of 64 bits (pairs of fp32 tell nearly always; fp64 itself takes 40 us a token).
// Bound by the latency of its steps and the instructions of K maxima over the warp: 8191
// tokens of 256 experts in 8 groups, 8 chosen, 23 us, of which tokens done again are 8 at the
// end; a token of 16 experts 2.2.  A grid that stays and takes tokens in turn took 33 us where
// this took 30 (its loop's registers).
// ===========================================================================
constexpr int kSelThreads = 128;
constexpr int kSelWarps = kSelThreads / 32;

struct SelArgs {
    int T, E, K, sigmoid, G, top_groups, group_top, renorm;
    float scale;
    const float *logits, *bias;
    int32_t *idx;
    float *gate;
};

// Keys as integers in the keys' order; NaN below every number, 0 is left for what is
// out of the choice.
__device__ __forceinline__ uint32_t key_code(float v) {
    if (isnan(v)) return 1u;
    const uint32_t b = __float_as_uint(v + 0.f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_of(uint32_t code) {  // of a number's code
    return __uint_as_float((code & 0x80000000u) ? code & 0x7fffffffu : ~code);
}
__device__ __forceinline__ unsigned long long key_code(double v) {
    if (isnan(v)) return 1ull;
    const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.0);
    return (b >> 63) ? ~b : b | 0x8000000000000000ull;
}
template <typename T> __device__ __forceinline__ T warp_most(T v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// What 32 bits may be off by, of a score s, in steps of 2^-24.  exp(d) / z: |d| of the
// subtraction's rounding, 4 of the exponential, 4 + 13 of its sum over 256, 3 of the quotient
// by a reciprocal.  1 / (1 + exp(-d)): the fast exponential's 4 + 2.4 |d| (2 + 1.18 |d| units in
// the last place), of which the share 1 - s arrives, 1 of the sum, 4 of the fast quotient.  Both:
// 1 of the key's rounding, 1 of a bound's (key and error added).  (Beyond |d| = 104 s is 0 or 1.)
// And 2^-126 at once: the fast quotient of a larger divisor is 0, smaller numbers have fixed steps.
__device__ __forceinline__ float score_err(bool sigmoid, float s, float d) {
    d = fminf(fabsf(d), 128.f);
    const float steps = sigmoid ? 7.f + (1.f - s) * (5.f + 2.5f * d) : 29.f + 1.1f * d;
    return fmaf(s * steps, 5.9604645e-8f, 0x1p-125f);
}
constexpr float kSumErr = 1.2e-7f;  // the bias' part of a key's and a bound's rounding; a sum's

// The same numbers give the same keys.
__device__ __forceinline__ bool same_key(const float *l, const float *bias, int e, int f) {
    return __float_as_uint(l[e]) == __float_as_uint(l[f]) &&
           __float_as_uint(bias[e]) == __float_as_uint(bias[f]);
}

// A warp's scratch; what 64 bits need takes the same place.
struct alignas(16) SelScratch {
    union {
        struct {
            float score[256], key[256], group[256];
        } f;
        struct {
            float2 value[256], group[256];
        } p;
        struct {
            double score[256], group[256];
        } d;
    };
    int16_t sel[264];
};

// ---- numbers in pairs of fp32 (x + y, |y| at most half a step of x): about 44 bits at
// fp32's rate, where fp64 runs at a sixtieth of it ------------------------------------

__device__ __forceinline__ float2 pair_sum(float a, float b) {  // exact, any order
    const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
    return make_float2(s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t)));
}
__device__ __forceinline__ float2 pair_norm(float a, float b) {  // |a| >= |b|
    const float s = __fadd_rn(a, b);
    return make_float2(s, __fsub_rn(b, __fsub_rn(s, a)));
}
__device__ __forceinline__ float2 pair_add(float2 a, float2 b) {
    const float2 s = pair_sum(a.x, b.x);
    return pair_norm(s.x, s.y + (a.y + b.y));
}
__device__ __forceinline__ float2 pair_div(float2 a, float2 b) {
    const float r = 1.f / b.x, q = a.x * r;
    const float rem = fmaf(-q, b.x, a.x) + (a.y - q * b.y);
    return pair_norm(q, rem * r);
}

// exp(x) for |x| <= 80, to 2^-40 of itself: exp(x) = 2^(k/16) exp(r), k the nearest whole
// number to 16 x / log 2, 2^(j/16) for j < 16 from a table (Tang's method, ACM TOMS 15, 1989),
// exp(r), |r| < 0.022, by its series, the terms beyond r^2 in one fp32 (below 2^-19 and
// so off by less than 2^-42).  log 2 / 16 in three parts, the first two of 12 bits, so that
// their products with k are exact.
__constant__ float2 kPairRoots[16] = {
    {0x1.000000p+0f, 0.f},
    {0x1.0b5586p+0f, 0x1.9f3122p-25f},
    {0x1.172b84p+0f, -0x1.c15742p-27f},
    {0x1.2387a6p+0f, 0x1.ceac48p-25f},
    {0x1.306fe0p+0f, 0x1.4636e2p-25f},
    {0x1.3dea64p+0f, 0x1.824684p-25f},
    {0x1.4bfdaep+0f, -0x1.593abcp-25f},
    {0x1.5ab07ep+0f, -0x1.5bd5ecp-27f},
    {0x1.6a09e6p+0f, 0x1.9fcef4p-26f},
    {0x1.7a1148p+0f, -0x1.829fd0p-25f},
    {0x1.8ace54p+0f, 0x1.15506ep-27f},
    {0x1.9c4918p+0f, 0x1.51f848p-27f},
    {0x1.ae89fap+0f, -0x1.a94b14p-26f},
    {0x1.c199bep+0f, -0x1.3d56b2p-27f},
    {0x1.d5818ep+0f, -0x1.822dbcp-27f},
    {0x1.ea4afap+0f, 0x1.52486cp-27f},
};
__device__ __forceinline__ float2 pair_exp(float2 x) {
    const float k = rintf(x.x * 0x1.715476p+4f);
    float2 r = pair_sum(fmaf(-k, 0x1.62e000p-5f, x.x), -k * 0x1.0be000p-19f);
    r = pair_norm(r.x, r.y + (x.y - k * 0x1.be8e7cp-31f));
    const float q = __fmul_rn(r.x, r.x), ql = fmaf(r.x, r.x, -q);
    const float more = q * r.x * fmaf(r.x, fmaf(r.x, fmaf(r.x, 1.f / 720, 1.f / 120), 1.f / 24), 1.f / 6);
    const float2 a = pair_norm(1.f, r.x), b = pair_norm(a.x, 0.5f * q);
    const float low = ((r.y + fmaf(r.x, r.y, 0.5f * ql)) + (a.y + b.y)) + more;
    const int n = (int)k;
    const float2 t = kPairRoots[n & 15];
    const float h = __fmul_rn(b.x, t.x);
    const float2 e = pair_norm(h, fmaf(b.x, t.x, -h) + fmaf(b.x, t.y, low * t.x));
    const float two = __uint_as_float((uint32_t)((n >> 4) + 127) << 23);
    return make_float2(e.x * two, e.y * two);
}

__device__ __forceinline__ unsigned long long key_code(float2 v) {
    const uint32_t hi = key_code(v.x);  // (NaN: nothing behind it counts)
    return (unsigned long long)hi << 32 | (hi == 1u ? 0u : key_code(isnan(v.y) ? 0.f : v.y));
}
__device__ __forceinline__ bool pair_less(float2 a, float2 b) {
    return a.x < b.x || (a.x == b.x && a.y < b.y);
}
// What a score in pairs may be off by, 16 times over.
constexpr float kPairErr = 0x1p-36f;

// Group g is one of the `top` with the largest values.
template <typename F>
__device__ __forceinline__ bool group_in(const F *value, int G, int top, int g) {
    const auto mine = key_code(value[g]);
    int before = 0;
    for (int h = 0; h < G; ++h) {
        const auto other = key_code(value[h]);
        before += other > mine || (other == mine && h < g);
    }
    return before < top;
}

// The score 1 / (1 + exp(-x)) in pairs; NaN stays.
__device__ __forceinline__ float2 pair_sigmoid(float x) {
    if (isnan(x)) return make_float2(x, 0.f);
    if (x < -80.f) return make_float2(0.f, 0.f);
    const float2 e = pair_exp(make_float2(-fminf(x, 80.f), 0.f)), t = pair_sum(1.f, e.x);
    return pair_div(make_float2(1.f, 0.f), pair_norm(t.x, t.y + e.y));
}

// The K <= 32 experts chosen are the right ones, but some keys lie near to each other:
// their order anew (sigmoid scores and a bias); false where pairs do not tell.
__device__ __noinline__ bool order_pairs(const SelArgs &a, const float *l, SelScratch &w, int lane) {
    const bool in = lane < a.K;
    const int e = w.sel[in ? lane : 0];
    const float x = l[e], b = a.bias[e];
    const float2 s = pair_sigmoid(x), t = pair_sum(s.x, b);
    const float2 key = isfinite(t.x) ? pair_norm(t.x, t.y + s.y) : make_float2(s.x + b, 0.f);
    const unsigned long long mine = key_code(key);
    int before = 0;
    bool clear = true;
    for (int k = 0; k < a.K; ++k) {
        const float2 y = make_float2(__shfl_sync(0xffffffffu, key.x, k), __shfl_sync(0xffffffffu, key.y, k));
        const float yx = __shfl_sync(0xffffffffu, x, k), yb = __shfl_sync(0xffffffffu, b, k);
        const int f = __shfl_sync(0xffffffffu, e, k);
        const unsigned long long other = key_code(y);
        before += other > mine || (other == mine && f < e);
        const bool same = __float_as_uint(yx) == __float_as_uint(x) && __float_as_uint(yb) == __float_as_uint(b);
        if (in && k != lane && !same && isfinite(y.x) && isfinite(key.x) &&
            fabsf((key.x - y.x) + (key.y - y.y)) <= 2.f * kPairErr * (1.f + 0x1p-8f * (fabsf(b) + fabsf(yb))))
            clear = false;
    }
    __syncwarp();
    if (in) w.sel[before] = (int16_t)e;
    __syncwarp();
    return __all_sync(0xffffffffu, clear);
}

// The token in pairs: its experts in w.sel; false where these do not tell either.
template <int NE>
__device__ __noinline__ bool select_pairs(const SelArgs &a, const float *l, SelScratch &w, int lane,
                                          float m) {
    // (a rare call finds its instructions far away: loops stay loops)
    const int e0 = lane * NE;
    const bool biased = a.bias != nullptr, by_score = !biased && a.group_top == 2 && a.G > 1;
    float2 z = make_float2(0.f, 0.f);
    __syncwarp();
#pragma unroll 1
    for (int e = lane; e < a.E; e += 32) {
        const float x = l[e], d = x - m;
        float2 s;
        if (a.sigmoid) {
            s = pair_sigmoid(x);
        } else {
            s = make_float2(isnan(d) ? d : 0.f, 0.f);
            if (d >= -80.f) s = pair_exp(pair_sum(x, -m));
            z = pair_add(z, s);
        }
        w.p.value[e] = s;
    }
    if (!a.sigmoid)
#pragma unroll 1
        for (int o = 16; o > 0; o >>= 1)
            z = pair_add(z, make_float2(__shfl_xor_sync(0xffffffffu, z.x, o),
                                        __shfl_xor_sync(0xffffffffu, z.y, o)));
    float err = 0.f;
#pragma unroll 1
    for (int e = lane; e < a.E; e += 32) {
        float2 s = w.p.value[e];
        if (!a.sigmoid) s = pair_div(s, z);
        const float b = biased ? a.bias[e] : 0.f;
        if (isfinite(b)) err = fmaxf(err, kPairErr * (fabsf(s.x) + 0x1p-8f * fabsf(b)));
        if (biased) {
            const float2 t = pair_sum(s.x, b);
            s = isfinite(t.x) ? pair_norm(t.x, t.y + s.y) : make_float2(s.x + b, 0.f);
        } else if (!by_score) {
            s = make_float2(l[e], 0.f);
        }
        w.p.value[e] = s;
    }
    err = warp_most(err) + 0x1p-100f;
    __syncwarp();
    bool clear = true;
    unsigned long long code[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i)
        code[i] = e0 + i >= a.E ? 0ull : by_score ? key_code(make_float2(l[e0 + i], 0.f))
                                                  : key_code(w.p.value[e0 + i]);
    if (a.G > 1) {
        const int gs = a.E / a.G;
        int P = 1;
        while (2 * P * a.G <= 32 && 2 * P <= gs) P <<= 1;
        const float2 none = make_float2(-INFINITY, 0.f);
#pragma unroll 1
        for (int g0 = 0; g0 < a.G; g0 += 32 / P) {
            const int g = g0 + lane / P;
            float2 t1 = none, t2 = none;
            auto take = [&](float2 k) {
                if (isnan(k.x)) k = none;
                if (pair_less(t1, k)) {
                    t2 = t1;
                    t1 = k;
                } else if (pair_less(t2, k)) {
                    t2 = k;
                }
            };
            if (g < a.G)
#pragma unroll 1
                for (int i = lane & (P - 1); i < gs; i += P) take(w.p.value[g * gs + i]);
#pragma unroll 1
            for (int o = 1; o < P; o <<= 1) {
                const float2 o1 = make_float2(__shfl_xor_sync(0xffffffffu, t1.x, o),
                                              __shfl_xor_sync(0xffffffffu, t1.y, o));
                const float2 o2 = make_float2(__shfl_xor_sync(0xffffffffu, t2.x, o),
                                              __shfl_xor_sync(0xffffffffu, t2.y, o));
                take(o1);
                take(o2);
            }
            if (g < a.G && (lane & (P - 1)) == 0) {
                float2 v = t1;
                if (a.group_top == 2)
                    v = isfinite(t1.x) && isfinite(t2.x)
                            ? pair_add(make_float2(0.5f * t1.x, 0.5f * t1.y), make_float2(0.5f * t2.x, 0.5f * t2.y))
                            : make_float2(t1.x + t2.x, 0.f);
                w.p.group[g] = v;
            }
        }
        __syncwarp();
        // the worst group kept, the best left out
        float2 low = make_float2(INFINITY, 0.f), high = none;
#pragma unroll 1
        for (int g0 = 0; g0 < a.G; g0 += 32) {
            const int g = g0 + lane;
            bool in = false;
            if (g < a.G) {
                in = group_in(w.p.group, a.G, a.top_groups, g);
                float2 x = w.p.group[g];
                if (isnan(x.x)) x = none;
                if (in && pair_less(x, low)) low = x;
                if (!in && pair_less(high, x)) high = x;
            }
            const uint32_t kept = __ballot_sync(0xffffffffu, in);
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                const int of_g = (e0 + i) / gs - g0;
                if (of_g >= 0 && of_g < 32 && !((kept >> of_g) & 1u)) code[i] = 0;
            }
        }
#pragma unroll 1
        for (int o = 16; o > 0; o >>= 1) {
            const float2 x = make_float2(__shfl_xor_sync(0xffffffffu, low.x, o),
                                         __shfl_xor_sync(0xffffffffu, low.y, o));
            const float2 y = make_float2(__shfl_xor_sync(0xffffffffu, high.x, o),
                                         __shfl_xor_sync(0xffffffffu, high.y, o));
            if (pair_less(x, low)) low = x;
            if (pair_less(high, y)) high = y;
        }
        if ((biased || by_score) && high.x > -INFINITY)
            clear = isfinite(low.x) && (low.x - high.x) + (low.y - high.y) > 2.f * err;
    }
#pragma unroll 1
    for (int k = 0; k < a.K; ++k) {
        unsigned long long best = code[0];
        int at = 0;
#pragma unroll
        for (int i = 1; i < NE; ++i)
            if (code[i] > best) {
                best = code[i];
                at = i;
            }
        const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32));
        const bool mine = (uint32_t)(best >> 32) == hi;
        const uint32_t lo = __reduce_max_sync(0xffffffffu, mine ? (uint32_t)best : 0u);
        const int who = __ffs(__ballot_sync(0xffffffffu, mine && (uint32_t)best == lo)) - 1;
        if (lane == who) {
            w.sel[k] = (int16_t)(e0 + at);
#pragma unroll
            for (int i = 0; i < NE; ++i)
                if (i == at) code[i] = 0;
        }
    }
    __syncwarp();
    if (biased) {
        // neighbours among the K; the last of them and each one left out that is not its equal
        auto apart = [&](int e, int f) {
            const float2 x = w.p.value[e], y = w.p.value[f];
            return !isfinite(x.x) || !isfinite(y.x) || (x.x - y.x) + (x.y - y.y) > 2.f * err ||
                   same_key(l, a.bias, e, f);
        };
        for (int k = lane; k + 1 < a.K; k += 32) clear = clear && apart(w.sel[k], w.sel[k + 1]);
        const int last = w.sel[a.K - 1];
#pragma unroll
        for (int i = 0; i < NE; ++i)
            if (code[i]) clear = clear && apart(last, e0 + i);
    }
    return __all_sync(0xffffffffu, clear);
}

// The token in 64 bits: any sizes, no haste (an equality that pairs leave open).
__device__ __noinline__ void select_exact(const SelArgs &a, const float *l, SelScratch &w, int lane) {
    double m = -INFINITY, z = 0;
    if (!a.sigmoid) {
        for (int e = lane; e < a.E; e += 32) m = fmax(m, (double)l[e]);
        m = warp_most(m);
        for (int e = lane; e < a.E; e += 32) {
            w.d.score[e] = exp((double)l[e] - m);
            z += w.d.score[e];
        }
        z = warp_sum(z);
    }
    for (int e = lane; e < a.E; e += 32) {
        const double s = a.sigmoid ? 1.0 / (1.0 + exp(-(double)l[e])) : w.d.score[e] / z;
        w.d.score[e] = s;
    }
    __syncwarp();
    auto key = [&](int e) { return a.bias ? w.d.score[e] + (double)a.bias[e] : (double)l[e]; };
    const int gs = a.E / a.G;
    uint32_t out = 0;  // of the experts lane, lane + 32, ...: those out of the choice
    if (a.G > 1) {
        const bool by_score = !a.bias && a.group_top == 2;
        for (int g = lane; g < a.G; g += 32) {
            double t1 = -INFINITY, t2 = -INFINITY;
            for (int i = 0; i < gs; ++i) {
                double k = by_score ? w.d.score[g * gs + i] : key(g * gs + i);
                if (isnan(k)) k = -INFINITY;
                t2 = fmax(t2, fmin(t1, k));
                t1 = fmax(t1, k);
            }
            w.d.group[g] = a.group_top == 2 ? t1 + t2 : t1;
        }
        __syncwarp();
        for (int i = 0, e = lane; e < a.E; ++i, e += 32)
            if (!group_in(w.d.group, a.G, a.top_groups, e / gs)) out |= 1u << i;
    }
    for (int k = 0; k < a.K; ++k) {
        unsigned long long best = 0;
        int at = 256;
        for (int i = 0, e = lane; e < a.E; ++i, e += 32) {
            const unsigned long long c = (out >> i) & 1u ? 0ull : key_code(key(e));
            if (c > best) {
                best = c;
                at = e;
            }
        }
        const unsigned long long top = warp_most(best);
        const int e = (int)__reduce_min_sync(0xffffffffu, best == top ? (unsigned)at : 256u);
        if ((e & 31) == lane) out |= 1u << (e >> 5);
        if (lane == 0) w.sel[k] = (int16_t)e;
    }
    __syncwarp();
}

__device__ void write_exact(const SelArgs &a, int t, const SelScratch &w, int lane) {
    double sum = 0;
    for (int k = lane; k < a.K; k += 32) sum += w.d.score[w.sel[k]];
    sum = warp_sum(sum);
    for (int k = lane; k < a.K; k += 32) {
        const double s = w.d.score[w.sel[k]];
        a.idx[(size_t)t * a.K + k] = w.sel[k];
        a.gate[(size_t)t * a.K + k] = (float)((a.renorm ? s / sum : s) * (double)a.scale);
    }
}

// 1 / (1 + exp(-x)), also where exp(-x) leaves the numbers of 32 bits.
__device__ __forceinline__ float sigmoid(float x) {
    const float e = expf(-fabsf(x));
    return (x < 0.f ? e : 1.f) / (1.f + e);
}

template <int NE>
__device__ __forceinline__ void keep(float *to, const float (&v)[NE]) {
    if constexpr (NE >= 4) {
#pragma unroll
        for (int i = 0; i < NE; i += 4)
            *reinterpret_cast<float4 *>(to + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < NE; ++i) to[i] = v[i];
    }
}

template <int NE>
__global__ void __launch_bounds__(kSelThreads)
k_select(const SelArgs a) {
    __shared__ SelScratch scratch[kSelWarps];
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t = blockIdx.x * kSelWarps + warp;
    if (t >= a.T) return;
    SelScratch &w = scratch[warp];
    const float *l = a.logits + (size_t)t * a.E;
    const int e0 = lane * NE;
    const bool biased = a.bias != nullptr, by_score = !biased && a.group_top == 2 && a.G > 1;
    float v[NE], s[NE], b[NE], m = 0.f, z = 1.f;
#pragma unroll
    for (int i = 0; i < NE; ++i) v[i] = -INFINITY;
    if (NE >= 4 && a.E % 4 == 0) {  // (rows of 16-byte multiples)
#pragma unroll
        for (int i = 0; i + 4 <= NE; i += 4)
            if (e0 + i < a.E) {
                const float4 f = *reinterpret_cast<const float4 *>(l + e0 + i);
                v[i] = f.x;
                v[i + 1] = f.y;
                v[i + 2] = f.z;
                v[i + 3] = f.w;
            }
    } else {
#pragma unroll
        for (int i = 0; i < NE; ++i)
            if (e0 + i < a.E) v[i] = l[e0 + i];
    }
#pragma unroll
    for (int i = 0; i < NE; ++i) b[i] = biased && e0 + i < a.E ? a.bias[e0 + i] : 0.f;
    if (!a.sigmoid) {
        m = v[0];
#pragma unroll
        for (int i = 1; i < NE; ++i) m = fmaxf(m, v[i]);
        m = warp_most(m);
        z = 0.f;
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            s[i] = e0 + i < a.E ? expf(v[i] - m) : 0.f;
            z += s[i];
        }
        z = moe::warp_sum(z);
        const float inv = 1.f / z;
#pragma unroll
        for (int i = 0; i < NE; ++i) s[i] *= inv;
    } else if (biased || by_score) {
#pragma unroll
        for (int i = 0; i < NE; ++i) s[i] = __fdividef(1.f, 1.f + __expf(-v[i]));
    }
    uint32_t code[NE];
    float err = 0.f, kv[NE], up[NE];  // the largest error, keys, keys with their errors
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        const float key = biased ? s[i] + b[i] : v[i];
        code[i] = e0 + i < a.E ? key_code(key) : 0u;
        kv[i] = key;
        up[i] = -INFINITY;
        if ((biased || by_score) && e0 + i < a.E && isfinite(key)) {
            const float off = score_err(a.sigmoid, s[i], v[i] - m) + kSumErr * fabsf(b[i]);
            err = fmaxf(err, off);
            up[i] = key + off;
        }
    }
    if (biased || by_score) keep<NE>(w.f.score + e0, s);
    keep<NE>(w.f.key + e0, kv);
    bool clear = true;
    if (a.G > 1) {
        const int gs = a.E / a.G;
        __syncwarp();
        // the two largest of each group: of a lane's own experts where it has no other group's
        // (those of a group are P lanes then), else through shared memory
        int P = gs / NE;
        const bool own_group = P * NE == gs && (P & (P - 1)) == 0;
        if (!own_group)
            for (P = 1; 2 * P * a.G <= 32 && 2 * P <= gs;) P <<= 1;
        const float *of = by_score ? w.f.score : w.f.key;
        for (int g0 = 0; g0 < a.G; g0 += own_group ? a.G : 32 / P) {
            const int g = g0 + lane / P;
            float t1 = -INFINITY, t2 = -INFINITY;
            auto take = [&](float k) {
                if (isnan(k)) k = -INFINITY;
                t2 = fmaxf(t2, fminf(t1, k));
                t1 = fmaxf(t1, k);
            };
            if (own_group) {
#pragma unroll
                for (int i = 0; i < NE; ++i) take(by_score ? s[i] : kv[i]);
            } else if (g < a.G) {
                for (int i = lane & (P - 1); i < gs; i += P) take(of[g * gs + i]);
            }
            for (int o = 1; o < P; o <<= 1) {
                const float o1 = __shfl_xor_sync(0xffffffffu, t1, o), o2 = __shfl_xor_sync(0xffffffffu, t2, o);
                t2 = fmaxf(fminf(t1, o1), fmaxf(t2, o2));
                t1 = fmaxf(t1, o1);
            }
            // (half the sum, which stays in range where both are the type's lowest)
            if (g < a.G && (lane & (P - 1)) == 0)
                w.f.group[g] = a.group_top == 2 ? 0.5f * t1 + 0.5f * t2 : t1;
        }
        __syncwarp();
        uint32_t low = 0xffffffffu, high = 0u;  // the worst kept, the best left out
        for (int g0 = 0; g0 < a.G; g0 += 32) {
            const int g = g0 + lane;
            bool in = false;
            if (g < a.G) {
                in = group_in(w.f.group, a.G, a.top_groups, g);
                const uint32_t c = key_code(w.f.group[g]);
                if (in) low = min(low, c);
                else high = max(high, c);
            }
            const uint32_t kept = __ballot_sync(0xffffffffu, in);
            if (own_group) {  // (32 groups at most)
                if (!((kept >> (lane / P)) & 1u))
#pragma unroll
                    for (int i = 0; i < NE; ++i) code[i] = 0u;
            } else {
#pragma unroll
                for (int i = 0; i < NE; ++i) {
                    const int of_g = (e0 + i) / gs - g0;
                    if (of_g >= 0 && of_g < 32 && !((kept >> of_g) & 1u)) code[i] = 0u;
                }
            }
        }
        if ((biased || by_score) && a.top_groups < a.G) {
            low = __reduce_min_sync(0xffffffffu, low);
            high = __reduce_max_sync(0xffffffffu, high);
            err = warp_most(err);
            // both sides off by up to a key (or the mean of two) and its rounding; NaN and minus
            // infinity are what they are in 64 bits too
            if (high > key_code(-INFINITY)) {
                const float lo = key_of(low), hi = key_of(high);
                clear = lo < INFINITY && lo - hi > 2.f * err + kSumErr * (fabsf(lo) + fabsf(hi));
            }
        }
    }
    for (int k = 0; k < a.K; ++k) {
        uint32_t best = code[0];
        int at = 0;
#pragma unroll
        for (int i = 1; i < NE; ++i)
            if (code[i] > best) {
                best = code[i];
                at = i;
            }
        const uint32_t top = __reduce_max_sync(0xffffffffu, best);
        // (the lowest lane has the lowest experts)
        const int who = __ffs(__ballot_sync(0xffffffffu, best == top)) - 1;
        if (lane == who) {
            w.sel[k] = (int16_t)(e0 + at);
#pragma unroll
            for (int i = 0; i < NE; ++i)
                if (i == at) code[i] = 0u;
        }
    }
    __syncwarp();
    // clear: which the K are; order: theirs is clear too
    bool order = true;
    if (biased) {
        float lo = INFINITY, hi = -INFINITY;  // the least that a key kept may be, the most of one left out
        auto off = [&](int e) {
            return score_err(a.sigmoid, w.f.score[e], l[e] - m) + kSumErr * fabsf(a.bias[e]);
        };
        for (int k = lane; k < a.K; k += 32) {
            const int e = w.sel[k];
            const float ke = w.f.key[e];
            if (!isfinite(ke)) continue;  // an infinite bias decides by itself; NaN is below everything
            lo = fminf(lo, ke - off(e));
            if (k + 1 == a.K) continue;
            const int f = w.sel[k + 1];
            const float kf = w.f.key[f];
            if (isfinite(kf) && !(ke - kf > off(e) + off(f)) && !same_key(l, a.bias, e, f)) order = false;
        }
#pragma unroll
        for (int i = 0; i < NE; ++i)
            if (code[i]) hi = fmaxf(hi, up[i]);
        const int last = w.sel[a.K - 1];
        const float kl = w.f.key[last];
        if (isfinite(kl)) {
            lo = key_of(__reduce_min_sync(0xffffffffu, key_code(lo)));
            hi = key_of(__reduce_max_sync(0xffffffffu, key_code(hi)));
            if (!(lo > hi)) {
                // Equals of the last one kept may be left out, by their index, where every other one kept
                // is above them and every other one left out is below those kept.
                bool fits = true, equal = false;
#pragma unroll
                for (int i = 0; i < NE; ++i)
                    if (code[i]) {
                        if (same_key(l, a.bias, last, e0 + i)) equal = true;
                        else if (!(lo > up[i])) fits = false;
                    }
                if (__any_sync(0xffffffffu, equal))
                    for (int k = lane; k < a.K; k += 32) {
                        const int e = w.sel[k];
                        const float ke = w.f.key[e];
                        if (isfinite(ke) && !(ke - off(e) > kl + off(last)) && !same_key(l, a.bias, last, e))
                            fits = false;
                    }
                if (!fits) clear = false;
            }
        }
    }
    clear = __all_sync(0xffffffffu, clear);
    order = __all_sync(0xffffffffu, order);
    if (clear && !order) clear = a.sigmoid && a.K <= 32 && order_pairs(a, l, w, lane);
    // weights: the scores anew, with the full exponential and quotient
    float sum = 0.f, own = 0.f;
    auto weights = [&]() {
        sum = 0.f;
        for (int k = lane; k < a.K; k += 32) {
            const float x = l[w.sel[k]];
            own = a.sigmoid ? sigmoid(x) : expf(x - m) / z;
            sum += own;
        }
        sum = moe::warp_sum(sum);
    };
    weights();
    // (a sum that 32 bits hold badly or not at all: 64 bits too)
    const bool tiny = a.renorm && sum < 1e-30f;
    if (!clear || tiny) {
        if (tiny || !select_pairs<NE>(a, l, w, lane, m)) {
            __syncwarp();
            select_exact(a, l, w, lane);
            write_exact(a, t, w, lane);
            return;
        }
        weights();
    }
    for (int k = lane; k < a.K; k += 32) {
        const int e = w.sel[k];
        if (a.K > 32) {
            const float x = l[e];
            own = a.sigmoid ? sigmoid(x) : expf(x - m) / z;
        }
        a.idx[(size_t)t * a.K + k] = e;
        a.gate[(size_t)t * a.K + k] = (a.renorm ? own / sum : own) * a.scale;
    }
}

// ---- host side ---------------------------------------------------------------

bool q_aligned(const void *p) { return p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool q_aligned_opt(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool q_dtype(int32_t v) { return v == MOE_F32 || v == MOE_BF16; }
moe_status q_status(cudaError_t e) { return e == cudaSuccess ? MOE_OK : MOE_ERR_CUDA; }

cudaError_t launch_rows(int rows, int cols, int K, const void *x, int32_t x_dtype,
                        const int32_t *inv, void *q, float *scale, int *count, int n_count,
                        cudaStream_t st) {
    // runs of 4 blocks where that leaves every SM several, else single blocks
    const int sms = device_info().sm_count, nb = q_blocks(cols);
    const bool runs = (long long)rows * nb >= (long long)sms * 128;
    const int U = runs ? 4 : 1;
    const long long items = (long long)rows * ((nb + U - 1) / U);
    const int grid = (int)std::max(1LL, std::min<long long>((items + kRowsThreads / 16 - 1) / (kRowsThreads / 16),
                                                            sms * 8LL));
    uint8_t *qp = static_cast<uint8_t *>(q);
    void *args[] = {&rows, &cols, &K, &x, &inv, &qp, &scale, &count, &n_count};
    LaunchScope ls("quant_rows", st);
    const void *kern = x_dtype == MOE_BF16
                           ? (runs ? (const void *)k_quant_rows<bf16, 4> : (const void *)k_quant_rows<bf16, 1>)
                           : (runs ? (const void *)k_quant_rows<float, 4> : (const void *)k_quant_rows<float, 1>);
    return launch_pdl(kern, dim3(grid), dim3(kRowsThreads), 0, st, args);
}

moe_status check_router(const moe_dims &d, const moe_router *r) {
    if (!r) return MOE_ERR_INVALID_ARG;
    if (r->score != MOE_SCORE_SOFTMAX && r->score != MOE_SCORE_SIGMOID) return MOE_ERR_INVALID_ARG;
    if (r->n_groups < 1 || r->n_groups > d.n_experts || d.n_experts % r->n_groups)
        return MOE_ERR_INVALID_ARG;
    const int gs = d.n_experts / r->n_groups;
    if (r->top_groups < 1 || r->top_groups > r->n_groups || r->top_groups * gs < d.top_k)
        return MOE_ERR_INVALID_ARG;
    if (r->group_top < 1 || r->group_top > 2 || (r->n_groups > 1 && r->group_top > gs))
        return MOE_ERR_INVALID_ARG;
    if (r->renormalise != 0 && r->renormalise != 1) return MOE_ERR_INVALID_ARG;
    if (!isfinite(r->scale)) return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

cudaError_t launch_select(const moe_dims &d, const moe_router &r, int T, const float *logits,
                          const float *bias, int32_t *idx, float *gate, cudaStream_t st) {
    SelArgs a{T, d.n_experts, d.top_k, r.score == MOE_SCORE_SIGMOID, r.n_groups, r.top_groups,
              r.group_top, r.renormalise, r.scale, logits, bias, idx, gate};
    void *args[] = {&a};
    const void *kern = d.n_experts <= 32    ? (const void *)k_select<1>
                       : d.n_experts <= 64  ? (const void *)k_select<2>
                       : d.n_experts <= 128 ? (const void *)k_select<4>
                                            : (const void *)k_select<8>;
    LaunchScope ls("route_select", st);
    return launch_pdl(kern, dim3((T + kSelWarps - 1) / kSelWarps), dim3(kSelThreads), 0, st, args);
}

// Workspace of the experts and the layer for T tokens.
struct QuantLayout {
    size_t idx, gate, logits, counts, offsets, perm, inv, x8, xs, h8, hs, y, part, count, total;
    int cols;
};
QuantLayout quant_layout(const moe_dims &d, int64_t T) {
    auto up = [](size_t v) { return (v + 255) & ~size_t(255); };
    const size_t S = (size_t)T * d.top_k;
    QuantLayout L{};
    size_t o = 0;
    L.cols = q_stream_cols(d.n_experts, (long long)S);
    L.idx = o; o += up(S * 4);
    L.gate = o; o += up(S * 4);
    L.logits = o; o += up((size_t)T * d.n_experts * 4);
    L.counts = o; o += up((size_t)d.n_experts * 4);
    L.offsets = o; o += up(((size_t)d.n_experts + 1) * 4);
    L.perm = o; o += up(S * 4);
    L.inv = o; o += up(S * 4);
    L.x8 = o; o += up(S * d.d_model);
    L.xs = o; o += up(S * q_blocks(d.d_model) * 4);
    L.h8 = o; o += up(S * d.ffn_hidden);
    L.hs = o; o += up(S * q_blocks(d.ffn_hidden) * 4);
    L.y = o; o += up(S * d.d_model * 4);
    L.part = o; o += up(q_part_floats(L.cols, true) * 4);
    L.count = o; o += up(2 * kQMaxCtas * 4);
    L.total = o;
    return L;
}

moe_status check_quant_dims(const moe_dims *d) {
    moe_status s = check_layer_dims(d);
    if (s != MOE_OK) return s;
    if (d->d_model % 16 || d->ffn_hidden % 16) return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

template <typename P> P *at(void *ws, size_t off) {
    return reinterpret_cast<P *>(static_cast<char *>(ws) + off);
}

bool experts_ok(const moe_quant_experts *w) {
    return w && q_aligned(w->w1) && q_aligned(w->v1) && q_aligned(w->w2) && q_aligned(w->w1_scale) &&
           q_aligned(w->v1_scale) && q_aligned(w->w2_scale);
}

// Rows enough for the kernel of many rows, whose units of up to 128 rows x 256 weight rows cost the
// same however few rows there are (us, streamed and by it).  More than 64 a group, where the
// streaming kernel takes a second tile (8192 x 6144: 2 groups of 80 44 and 28, 8 of 100 145 and
// 74); of a single matrix, whose units are few, more than 128 (8192 x 6144: 128 rows 26 and 26, 144
// rows 35 and 26; 1024 x 8192: 128 rows 19 and 33).  From 34 on where the units go twice around
// (16 experts of 6144 x 10752: 24 to 40 rows 505 to 513 and 498 to 507; 40 of 2000 x 1424: 30 rows
// 107 and 99, 45 rows 109 and 100; but 6 groups of 40 rows, 8192 x 6144, 192 units on 152 SMs: 63
// and 66).
bool many_rows(int E, long long S, int n_out) {
    if (E == 1) return S > 128;
    return S > 64LL * E ||
           (S >= 34LL * E && (long long)E * ((n_out + 511) / 512) >= device_info().sm_count);
}

// The experts' products of slots that are dispatched already, and their combine.
cudaError_t quant_experts(const moe_dims &d, int T, const void *x, const moe_quant_experts &w,
                          const float *gate, const QuantLayout &L, void *ws, const void *residual,
                          void *out, cudaStream_t st) {
    const int S = T * d.top_k, D = d.d_model, F = d.ffn_hidden, E = d.n_experts;
    const int32_t *offsets = at<int32_t>(ws, L.offsets), *inv = at<int32_t>(ws, L.inv);
    int *count = at<int>(ws, L.count);
    cudaError_t e = launch_rows(T, D, d.top_k, x, d.x_dtype, inv, at<void>(ws, L.x8),
                                at<float>(ws, L.xs), count, 2 * kQMaxCtas, st);
    if (e != cudaSuccess) return e;
    const QuantGemm gu{E, S, D, F, offsets, at<void>(ws, L.x8), at<float>(ws, L.xs)};
    const QuantUp up{w.w1, w.v1, w.w1_scale, w.v1_scale, at<void>(ws, L.h8), at<float>(ws, L.hs)};
    const QuantGemm gd{E, S, F, D, offsets, at<void>(ws, L.h8), at<float>(ws, L.hs)};
    const QuantDown down{w.w2, w.w2_scale, at<void>(ws, L.y), 0};
    const QuantParts pu{at<float>(ws, L.part), count}, pd{at<float>(ws, L.part), count + kQMaxCtas};
    if (many_rows(E, S, D)) {
        e = launch_quant_wide_up(gu, up, st);
        if (e == cudaSuccess) e = launch_quant_wide_down(gd, down, st);
    } else {
        e = launch_quant_stream_up(gu, up, pu, L.cols, st);
        if (e == cudaSuccess) e = launch_quant_stream_down(gd, down, pd, L.cols, false, st);
    }
    if (e == cudaSuccess)
        e = launch_layer_combine(d, T, at<float>(ws, L.y), inv, gate, residual, out, st);
    return e;
}

// Workspace of a product for up to S rows: scales, counters, parts.
struct ProductLayout {
    size_t xs, count, part, total;
    int cols;
};
ProductLayout product_layout(int E, int n_in, int S) {
    auto up = [](size_t v) { return (v + 255) & ~size_t(255); };
    ProductLayout L{};
    L.cols = q_stream_cols(E, S);
    size_t o = 0;
    L.xs = o; o += up((size_t)S * q_blocks(n_in) * 4);
    L.count = o; o += up(kQMaxCtas * 4);
    L.part = o; o += up(q_part_floats(L.cols, false) * 4);
    L.total = o;
    return L;
}

moe_status check_product(int32_t E, int32_t n_out, int32_t n_in, int32_t S) {
    if (E < 1 || E > 256 || n_out < 8 || n_out > 65536 || n_out % 8 || n_in < 16 || n_in > 65536 ||
        n_in % 16 || S < 0 || S > (1 << 24))
        return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

moe_status moe_quantize_rows(int32_t rows, int32_t cols, const void *x, int32_t x_dtype, void *q,
                             float *scale, moe_stream_t stream) {
    MOE_INJECT("moe_quantize_rows");
    if (rows < 0 || rows > (1 << 24) || cols < 16 || cols > 65536 || cols % 16 || !q_dtype(x_dtype))
        return MOE_ERR_INVALID_ARG;
    if (rows == 0) return MOE_OK;
    if (!q_aligned(x) || !q_aligned(q) || !q_aligned(scale)) return MOE_ERR_INVALID_ARG;
    return q_status(launch_rows(rows, cols, 0, x, x_dtype, nullptr, q, scale, nullptr, 0,
                                (cudaStream_t)stream));
}

moe_status moe_quantize_blocks(int32_t n, int32_t rows, int32_t cols, const void *w, int32_t w_dtype,
                               void *q, float *scale, moe_stream_t stream) {
    MOE_INJECT("moe_quantize_blocks");
    if (n < 0 || n > 256 || rows < 8 || rows > 65536 || rows % 8 || cols < 16 || cols > 65536 ||
        cols % 16 || !q_dtype(w_dtype))
        return MOE_ERR_INVALID_ARG;
    if (n == 0) return MOE_OK;
    if (!q_aligned(w) || !q_aligned(q) || !q_aligned(scale)) return MOE_ERR_INVALID_ARG;
    const unsigned grid = (unsigned)n * q_blocks(rows) * q_blocks(cols);
    LaunchScope ls("quant_blocks", (cudaStream_t)stream);
    uint8_t *qp = static_cast<uint8_t *>(q);
    if (w_dtype == MOE_BF16)
        k_quant_blocks<bf16><<<grid, 256, 0, (cudaStream_t)stream>>>(
            rows, cols, static_cast<const bf16 *>(w), qp, scale);
    else
        k_quant_blocks<float><<<grid, 256, 0, (cudaStream_t)stream>>>(
            rows, cols, static_cast<const float *>(w), qp, scale);
    return q_status(cudaGetLastError());
}

moe_status moe_route_select(const moe_dims *dims, const moe_router *router, int32_t T,
                            const float *logits, const float *bias_opt, int32_t *topk_idx,
                            float *topk_gate, moe_stream_t stream) {
    MOE_INJECT("moe_route_select");
    moe_status s = check_layer_dims(dims);
    if (s == MOE_ERR_UNSUPPORTED) s = MOE_OK;  // (only E and K count here)
    if (s != MOE_OK) return s;
    if ((s = check_router(*dims, router)) != MOE_OK) return s;
    if ((s = check_layer_tokens(dims, T)) != MOE_OK) return s;
    if (T == 0) return MOE_OK;
    if (!q_aligned(logits) || !q_aligned_opt(bias_opt) || !topk_idx || !topk_gate)
        return MOE_ERR_INVALID_ARG;
    return q_status(launch_select(*dims, *router, T, logits, bias_opt, topk_idx, topk_gate,
                                  (cudaStream_t)stream));
}

moe_status moe_quant_product_workspace_size(int32_t n_groups, int32_t n_out, int32_t n_in,
                                            int32_t max_rows, size_t *bytes) {
    moe_status s = check_product(n_groups, n_out, n_in, max_rows);
    if (s != MOE_OK) return s;
    if (!bytes) return MOE_ERR_INVALID_ARG;
    *bytes = product_layout(n_groups, n_in, max_rows).total;
    return MOE_OK;
}

moe_status moe_quant_product(int32_t n_groups, int32_t n_out, int32_t n_in, int32_t S, const void *x,
                             const float *x_scale, const int32_t *offsets_opt, const void *w,
                             const float *w_scale, void *y, int32_t y_dtype, void *ws,
                             size_t ws_bytes, moe_stream_t stream) {
    MOE_INJECT("moe_quant_product");
    moe_status s = check_product(n_groups, n_out, n_in, S);
    if (s != MOE_OK) return s;
    if (!q_dtype(y_dtype) || (n_groups > 1 && !offsets_opt)) return MOE_ERR_INVALID_ARG;
    if (S == 0) return MOE_OK;
    if (!q_aligned(x) || !q_aligned(x_scale) || !q_aligned(w) || !q_aligned(w_scale) || !q_aligned(y))
        return MOE_ERR_INVALID_ARG;
    const ProductLayout L = product_layout(n_groups, n_in, S);
    if (!q_aligned(ws) || ws_bytes < L.total) return MOE_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    int *count = at<int>(ws, L.count);
    float *xs = at<float>(ws, L.xs);
    {
        int nb = q_blocks(n_in), n = kQMaxCtas;
        void *args[] = {&S, &nb, &x_scale, &xs, &count, &n};
        LaunchScope ls("quant_scales", st);
        if (launch_pdl((const void *)k_quant_scales,
                       dim3(std::min((S + 31) / 32, 1024), (nb + 31) / 32), dim3(256), 0, st,
                       args) != cudaSuccess)
            return MOE_ERR_CUDA;
    }
    const QuantGemm g{n_groups, S, n_in, n_out, offsets_opt, x, xs};
    const QuantDown down{w, w_scale, y, y_dtype == MOE_BF16};
    if (many_rows(n_groups, S, n_out))
        return q_status(launch_quant_wide_down(g, down, st));
    return q_status(launch_quant_stream_down(g, down, QuantParts{at<float>(ws, L.part), count}, L.cols,
                                             true, st));
}

moe_status moe_quant_workspace_size(const moe_dims *dims, int32_t max_tokens, size_t *bytes) {
    moe_status s = check_quant_dims(dims);
    if (s == MOE_ERR_UNSUPPORTED) s = MOE_OK;  // sizing does not depend on dtypes
    if (s != MOE_OK) return s;
    if (!bytes || max_tokens < 0) return MOE_ERR_INVALID_ARG;
    if ((s = check_layer_tokens(dims, max_tokens)) != MOE_OK) return s;
    *bytes = quant_layout(*dims, max_tokens).total;
    return MOE_OK;
}

moe_status moe_quant_experts_forward(const moe_dims *dims, int32_t T, const void *x,
                                     const int32_t *topk_idx, const float *topk_gate,
                                     const moe_quant_experts *experts, const void *residual_opt,
                                     void *out, void *ws, size_t ws_bytes, moe_stream_t stream) {
    MOE_INJECT("moe_quant_experts_forward");
    moe_status s = check_quant_dims(dims);
    if (s != MOE_OK) return s;
    if ((s = check_layer_tokens(dims, T)) != MOE_OK) return s;
    if (T == 0) return MOE_OK;
    if (!q_aligned(x) || !topk_idx || !topk_gate || !experts_ok(experts) ||
        !q_aligned_opt(residual_opt) || !q_aligned(out))
        return MOE_ERR_INVALID_ARG;
    const QuantLayout L = quant_layout(*dims, T);
    if (!q_aligned(ws) || ws_bytes < L.total) return MOE_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = launch_layer_dispatch(*dims, T, topk_idx, at<int32_t>(ws, L.counts),
                                          at<int32_t>(ws, L.offsets), at<int32_t>(ws, L.perm),
                                          at<int32_t>(ws, L.inv), st);
    if (e == cudaSuccess)
        e = quant_experts(*dims, T, x, *experts, topk_gate, L, ws, residual_opt, out, st);
    return q_status(e);
}

moe_status moe_quant_layer_forward(const moe_dims *dims, const moe_router *router_opt, int32_t T,
                                   const void *x, const void *w_router, const float *bias_opt,
                                   const moe_quant_experts *experts, const void *residual_opt,
                                   void *out, void *ws, size_t ws_bytes, moe_stream_t stream) {
    MOE_INJECT("moe_quant_layer_forward");
    moe_status s = check_quant_dims(dims);
    if (s != MOE_OK) return s;
    if (router_opt && (s = check_router(*dims, router_opt)) != MOE_OK) return s;
    if (!router_opt && bias_opt) return MOE_ERR_INVALID_ARG;
    if ((s = check_layer_tokens(dims, T)) != MOE_OK) return s;
    if (T == 0) return MOE_OK;
    if (!q_aligned(x) || !q_aligned(w_router) || !q_aligned_opt(bias_opt) || !experts_ok(experts) ||
        !q_aligned_opt(residual_opt) || !q_aligned(out))
        return MOE_ERR_INVALID_ARG;
    const QuantLayout L = quant_layout(*dims, T);
    if (!q_aligned(ws) || ws_bytes < L.total) return MOE_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    int32_t *idx = at<int32_t>(ws, L.idx);
    float *gate = at<float>(ws, L.gate);
    float *logits = at<float>(ws, L.logits);
    int32_t *counts = at<int32_t>(ws, L.counts), *offsets = at<int32_t>(ws, L.offsets);
    int32_t *perm = at<int32_t>(ws, L.perm), *inv = at<int32_t>(ws, L.inv);
    cudaError_t e;
    if (!router_opt) {
        e = launch_layer_route_dispatch(*dims, T, x, w_router, idx, gate, counts, offsets, perm, inv,
                                        st);
    } else {
        e = launch_layer_route(*dims, T, x, w_router, logits, idx, gate, st);
        if (e == cudaSuccess) e = launch_select(*dims, *router_opt, T, logits, bias_opt, idx, gate, st);
        if (e == cudaSuccess)
            e = launch_layer_dispatch(*dims, T, idx, counts, offsets, perm, inv, st);
    }
    if (e == cudaSuccess) e = quant_experts(*dims, T, x, *experts, gate, L, ws, residual_opt, out, st);
    return q_status(e);
}

}  // extern "C"
