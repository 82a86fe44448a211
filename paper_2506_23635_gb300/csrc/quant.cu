// 8-bit experts: quantisation in blocks of 128, the choice of experts from logits, and
// the C ABI of the grouped products and of the layer over them (include/moe.h).
#include <math.h>

#include "quant.cuh"

namespace moe {
namespace {

// ===========================================================================
// Quantising rows: 16 lanes take a block of 128 numbers, eight each.  Bound by memory.
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
// they were loaded.
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
// The choice of experts: one warp a token.  Scores and keys in 32 bits first; where two
// of the keys that decide lie nearer to each other than the error of 32 bits, the warp
// does the token again in 64 bits, so that the choice is that of 64 bits.
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
__device__ __forceinline__ unsigned long long key_code(double v) {
    if (isnan(v)) return 1ull;
    const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.0);
    return (b >> 63) ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ uint32_t warp_max(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }
__device__ __forceinline__ unsigned long long warp_max(unsigned long long v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
template <typename F> struct CodeOf;
template <> struct CodeOf<float> { typedef uint32_t type; };
template <> struct CodeOf<double> { typedef unsigned long long type; };

__device__ __forceinline__ float sel_exp(float v) { return expf(v); }
__device__ __forceinline__ double sel_exp(double v) { return exp(v); }
template <typename F> __device__ __forceinline__ F warp_sum_of(F v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// What 32 bits may be off by: of a score s = exp(d) / z or 1 / (1 + exp(d)), in units of
// 2^-24: |d| of the subtraction's rounding, 4 of the exponential, 13 of the sum over 256,
// 2 of the sum and the quotient, doubled for second orders below; of a key, its rounding.
__device__ __forceinline__ float score_err(float s, float d) {
    return s * ((24.f + fabsf(d)) * 5.9604645e-8f);
}

template <typename F>
struct SelWarp {
    F score[256], key[256];
    F group[256];  // values of the groups
    int sel[257];
};

// The K (and one more) experts of a token with the largest keys in F's precision;
// false where 32 bits do not tell.
template <int NE, typename F>
__device__ bool select_token(const SelArgs &a, const float *l, SelWarp<F> &w, int lane) {
    typedef typename CodeOf<F>::type Code;
    constexpr bool kApprox = sizeof(F) == 4;
    F v[NE], m = -INFINITY;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        const int e = i * 32 + lane;
        v[i] = e < a.E ? (F)l[e] : (F)-INFINITY;
        m = fmax(m, v[i]);
    }
    F s[NE], err = 0;
    if (a.sigmoid) {
        m = 0;
#pragma unroll
        for (int i = 0; i < NE; ++i) s[i] = (F)1 / ((F)1 + sel_exp(-v[i]));
    } else {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
        F z = 0;
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            s[i] = i * 32 + lane < a.E ? sel_exp(v[i] - m) : (F)0;
            z += s[i];
        }
        z = warp_sum_of(z);
#pragma unroll
        for (int i = 0; i < NE; ++i) s[i] /= z;
    }
    Code code[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        const int e = i * 32 + lane;
        code[i] = 0;
        if (e < a.E) {
            const F key = a.bias ? s[i] + (F)a.bias[e] : v[i];
            code[i] = key_code(key);
            w.score[e] = s[i];
            w.key[e] = key;
            if (kApprox && a.G > 1)
                err = fmax(err, (F)score_err((float)s[i], (float)(v[i] - m)) +
                                    (a.bias ? (F)1.2e-7f * fabs((F)a.bias[e]) : (F)0));
        }
    }
    __syncwarp();
    bool clear = true;
    if (a.G > 1) {
        const int gs = a.E / a.G;
        int P = 1;
        while (2 * P * a.G <= 32) P <<= 1;
        const bool by_score = !a.bias && a.group_top == 2;
        if (kApprox)
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) err = fmax(err, __shfl_xor_sync(0xffffffffu, err, o));
        for (int g0 = 0; g0 < a.G; g0 += 32 / P) {
            const int g = g0 + lane / P;
            F t1 = -INFINITY, t2 = -INFINITY;
            if (g < a.G)
                for (int i = lane % P; i < gs; i += P) {
                    F k = by_score ? w.score[g * gs + i] : w.key[g * gs + i];
                    if (isnan(k)) k = -INFINITY;
                    t2 = fmax(t2, fmin(t1, k));
                    t1 = fmax(t1, k);
                }
            for (int o = 1; o < P; o <<= 1) {
                const F o1 = __shfl_xor_sync(0xffffffffu, t1, o), o2 = __shfl_xor_sync(0xffffffffu, t2, o);
                t2 = fmax(fmin(t1, o1), fmax(t2, o2));
                t1 = fmax(t1, o1);
            }
            if (g < a.G && lane % P == 0) w.group[g] = a.group_top == 2 ? t1 + t2 : t1;
        }
        __syncwarp();
        // a group's rank: how many are before it
        uint32_t out = 0;  // of this lane's experts
        F low = INFINITY, high = -INFINITY;  // the worst kept, the best left out
        for (int g0 = 0; g0 < a.G; g0 += 32) {
            const int g = g0 + lane;
            bool in = false;
            if (g < a.G) {
                const F mine = w.group[g];
                const Code cm = key_code(mine);
                int before = 0;
                for (int h = 0; h < a.G; ++h) {
                    const Code ch = key_code(w.group[h]);
                    before += ch > cm || (ch == cm && h < g);
                }
                in = before < a.top_groups;
                const F x = isnan(mine) ? (F)-INFINITY : mine;
                if (in) low = fmin(low, x);
                else high = fmax(high, x);
            }
            const uint32_t kept = __ballot_sync(0xffffffffu, in);
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                const int e = i * 32 + lane, of = e / gs - g0;
                if (e < a.E && of >= 0 && of < 32 && !((kept >> of) & 1u)) out |= 1u << i;
            }
        }
#pragma unroll
        for (int i = 0; i < NE; ++i)
            if ((out >> i) & 1u) code[i] = 0;
        if (kApprox && (a.bias || a.group_top == 2) && a.top_groups < a.G) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                low = fmin(low, __shfl_xor_sync(0xffffffffu, low, o));
                high = fmax(high, __shfl_xor_sync(0xffffffffu, high, o));
            }
            // both sides off by up to two keys each and their sum's rounding (infinite
            // values are exact)
            if (high > -INFINITY)
                clear = low < INFINITY &&
                        low - high > 4 * err + (F)1.2e-7f * (fabs(low) + fabs(high));
        }
    }
    const int n = kApprox && a.bias ? a.K + 1 : a.K;
    for (int k = 0; k < n; ++k) {
        Code best = code[0];
        int at = lane;
#pragma unroll
        for (int i = 1; i < NE; ++i)
            if (code[i] > best) {
                best = code[i];
                at = i * 32 + lane;
            }
        const Code top = warp_max(best);
        if (top == 0) {  // none is left (only for the one beyond K)
            if (lane == 0) w.sel[k] = -1;
            break;
        }
        const int e = (int)__reduce_min_sync(0xffffffffu, best == top ? (unsigned)at : 0xffffffffu);
#pragma unroll
        for (int i = 0; i < NE; ++i)
            if (i * 32 + lane == e) code[i] = 0;
        if (lane == 0) w.sel[k] = e;
    }
    __syncwarp();
    if (kApprox && a.bias)
        for (int k = lane; k < a.K; k += 32) {
            const int e = w.sel[k], f = w.sel[k + 1];
            if (f < 0) break;
            const float le = l[e], lf = l[f], be = a.bias[e], bf = a.bias[f];
            // the same numbers give the same keys
            if (__float_as_uint(le) == __float_as_uint(lf) && __float_as_uint(be) == __float_as_uint(bf))
                continue;
            const float ke = (float)w.key[e], kf = (float)w.key[f];
            // an infinite bias or none decides by itself; NaN is below everything
            if (isnan(ke) || isnan(kf) || isinf(ke) || isinf(kf)) continue;
            const float off = score_err((float)w.score[e], le - (float)m) +
                              score_err((float)w.score[f], lf - (float)m) +
                              1.2e-7f * (fabsf(be) + fabsf(bf));
            if (!(ke - kf > off)) clear = false;
        }
    return __all_sync(0xffffffffu, clear);
}

template <typename F>
__device__ void write_choice(const SelArgs &a, int t, SelWarp<F> &w, int lane) {
    F sum = 0;
    for (int k = lane; k < a.K; k += 32) sum += w.score[w.sel[k]];
    sum = warp_sum_of(sum);
    for (int k = lane; k < a.K; k += 32) {
        const int e = w.sel[k];
        const F s = w.score[e];
        a.idx[(size_t)t * a.K + k] = e;
        a.gate[(size_t)t * a.K + k] = (float)((a.renorm ? s / sum : s) * (F)a.scale);
    }
}

template <int NE>
__global__ void __launch_bounds__(kSelThreads)
k_select(const SelArgs a) {
    __shared__ SelWarp<float> sw[kSelWarps];
    __shared__ SelWarp<double> dw[1];
    __shared__ int redo[kSelWarps];
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t = blockIdx.x * kSelWarps + warp;
    bool again = false;
    if (t < a.T) {
        again = !select_token<NE, float>(a, a.logits + (size_t)t * a.E, sw[warp], lane);
        // weights whose sum 32 bits hold badly or not at all
        if (!again && a.renorm) {
            float sum = 0.f;
            for (int k = lane; k < a.K; k += 32) sum += sw[warp].score[sw[warp].sel[k]];
            again = warp_sum(sum) < 1e-30f;
        }
        if (!again) write_choice(a, t, sw[warp], lane);
    }
    if (lane == 0) redo[warp] = again;
    __syncthreads();
    // (rare: one warp after another, in one warp's worth of 64-bit scratch)
    if (warp == 0)
        for (int i = 0; i < kSelWarps; ++i)
            if (redo[i]) {
                const int u = blockIdx.x * kSelWarps + i;
                select_token<NE, double>(a, a.logits + (size_t)u * a.E, dw[0], lane);
                write_choice(a, u, dw[0], lane);
                __syncwarp();
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

// Rows enough for the CTA pairs.
bool many_rows(int E, long long S) { return S >= 128LL * E; }

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
    if (many_rows(E, S) && quant_pair_ok()) {
        e = launch_quant_pair_up(gu, up, st);
        if (e == cudaSuccess) e = launch_quant_pair_down(gd, down, st);
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
    if (many_rows(n_groups, S) && quant_pair_ok())
        return q_status(launch_quant_pair_down(g, down, st));
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
