// A paged key/value cache in 8 bits: appending to it, and its entry points.
//
// Keys and values lie as e4m3 numbers in pages [n_pages, Hkv, page_size, 128],
// a scale for each (page, key/value head): value = scale x number.  (The
// paper's inference keeps its cache in bf16, Sec. 5.1, and prints nothing of
// its layout.)
//
// k_paged_append: rows of a QKV projection -> rotated queries in bf16, rotated
// keys and values quantised into their pages.  For the rows of one page and
// head in a call, a = max |x| over them:
//   need  = the smallest 2^e >= a / 448, e >= -100
//   scale = need where the call writes the page's first position, otherwise
//           max(old scale, need); the page's other rows follow a larger scale
// Powers of two: e4m3 is a floating type, so a finer scale would move only where
// its range ends, not how it rounds; with them the division is exact, a page
// that grows rounds its earlier rows again only below the normal range, and
// the values in a 16-bit type are exact.
#include <math.h>

#include <algorithm>

#include "attn_plan.cuh"
#include "paged.cuh"

namespace moe {
namespace {

// Rotary angles: pair i of position p turns by p base^(-2i/128) =
// 2 pi (p r_i), r_i in turns as a 64-bit fixed-point fraction, so that p r_i
// modulo one turn is a product of integers (no 64-bit floating point, of which
// the SMs do little); its upper 32 bits are the angle to 2^-32 of a turn.
struct RopeTurns {
    uint64_t r[kPagedDh / 2];
};

// (64 powers take longer than a launch: a thread keeps those of its last base)
const RopeTurns &rope_turns(float base) {
    static thread_local RopeTurns t;
    static thread_local float of = 0.f;
    if (of == base) return t;
    of = base;
    for (int i = 0; i < kPagedDh / 2; ++i)
        t.r[i] = (uint64_t)llrint(pow((double)base, -2.0 * i / (double)kPagedDh) /
                                  6.283185307179586 * 9223372036854775808.0)
                 << 1;
    return t;
}

__device__ __forceinline__ void rope_sincos(uint64_t r, int p, float &sn, float &cs) {
    const int32_t turns = (int32_t)(((uint64_t)(uint32_t)p * r) >> 32);  // [-1/2, 1/2) x 2^32
    sincospif((float)turns * 4.656612873077393e-10f, &sn, &cs);          // x 2^-31: in half turns
}

// The projection's rows: bf16, fp32, or fp32 partial sums that are added in
// order.
enum : int { kInBf16 = 0, kInF32 = 1, kInParts = 2 };

struct QkvRows {
    const void *p;
    int width;  // (Hq + 2 Hkv) 128
    int T;
    int n_part;  // kInParts: parts of each row, 0: as many as `split` says
    long long part_stride;
    ProjSplit split;
};

// Elements i .. i + 3 (a) and i + 64 .. i + 67 (b) of head row hr of token t.
template <int IN>
__device__ __forceinline__ void load_pairs(const QkvRows &x, int t, int hr, int i, float (&a)[4],
                                           float (&b)[4]) {
    const size_t at = (size_t)t * x.width + (size_t)hr * kPagedDh + i;
    if constexpr (IN == kInBf16) {
        const bf16 *p = static_cast<const bf16 *>(x.p) + at;
        const uint2 u = __ldg(reinterpret_cast<const uint2 *>(p));
        const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p + kPagedDh / 2));
        unpack_bf16x2(u.x, a[0], a[1]);
        unpack_bf16x2(u.y, a[2], a[3]);
        unpack_bf16x2(v.x, b[0], b[1]);
        unpack_bf16x2(v.y, b[2], b[3]);
    } else {
        const float *p = static_cast<const float *>(x.p) + at;
        const int n = IN == kInF32    ? 1
                      : x.n_part > 0 ? x.n_part
                                     : x.split.parts(x.T, t, hr * kPagedDh);
        for (int k = 0; k < n; ++k) {
            const float4 u = __ldg(reinterpret_cast<const float4 *>(p + k * x.part_stride));
            const float4 v =
                __ldg(reinterpret_cast<const float4 *>(p + k * x.part_stride + kPagedDh / 2));
            const float w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] = k ? a[e] + w[e] : w[e];
                b[e] = k ? b[e] + w[4 + e] : w[4 + e];
            }
        }
    }
}

// The smallest power of two that holds magnitudes up to a (finite, >= 0).
__device__ __forceinline__ float scale_for(float a) {
    // a = m 2^x, 1 <= m < 2; 448 = 1.75 x 2^8
    const uint32_t b = __float_as_uint(a);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)(max(e, kPagedMinExp) + 127) << 23);
}

__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a <= 3.402823466e38f ? a : 0.f;
}
// What is stored of x: an infinity is a NaN (e4m3 has none; 448 would be a
// number that nobody gave).
__device__ __forceinline__ float storable(float x) {
    return fabsf(x) <= 3.402823466e38f ? x : __uint_as_float(0x7fffffffu);
}

constexpr int kAppThreads = 256;
constexpr int kAppHalves = kAppThreads / 16;  // half a warp takes a row, four pairs a lane
constexpr int kAppQTokens = 4;                // tokens of a block of the queries' part
constexpr int kAppGroup = 128;  // tokens among which a block looks for its pages' first ones
constexpr int kAppRows = 16;    // key and value rows of a block at most

// The pair's rotation.
__device__ __forceinline__ void turn(float &a, float &b, float sn, float cs) {
    const float u = a, v = b;
    a = u * cs - v * sn;
    b = v * cs + u * sn;
}

// Four numbers x / scale, as they are stored.
__device__ __forceinline__ uint32_t quantise(const float (&x)[4], float scale) {
    const float inv = 1.f / scale;
    const bool pow2 = (__float_as_uint(scale) & 0x7fffffu) == 0;
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = storable(pow2 ? x[e] * inv : x[e] / scale);
    return e4m3x2(y[0], y[1]) | e4m3x2(y[2], y[3]) << 16;
}

// Four stored numbers times ratio, rounded again.
__device__ __forceinline__ uint32_t rescale(uint32_t v, float ratio) {
    const float2 f0 = e4m3x2_to_float2(v & 0xffffu), f1 = e4m3x2_to_float2(v >> 16);
    return e4m3x2(f0.x * ratio, f0.y * ratio) | e4m3x2(f1.x * ratio, f1.y * ratio) << 16;
}

// The n-th set bit of four words.
__device__ __forceinline__ int nth_bit(const uint32_t (&w)[kAppGroup / 32], int n) {
    int at = 0;
#pragma unroll
    for (int i = 0; i < kAppGroup / 32; ++i) {
        const int c = __popc(w[i]);
        if (n >= 0 && n < c) at = i * 32 + (int)__fns(w[i], 0, n + 1);
        n -= c;
    }
    return at;
}

// Blocks [0, n_qb): queries, kAppHalves head rows of kAppQTokens tokens, half a
// warp a row.  The others: keys and values.  The tokens of a call that lie in one
// page are found from the first of them: a token leads its page if no earlier
// token of the call lies there.  Only one that does not follow its
// predecessor inside the page can (a start); starts look through the whole
// call's tokens, which may come in any order.  Blocks (group of 128 tokens, rows
// [rb rpb, (rb + 1) rpb) of the 2 Hkv key and value rows, slot): the starts of the
// group are shared out among its slots.  A page with one token of the call
// (decode): half a warp for each of the block's rows; else row by row, the
// page's tokens in registers between their maximum and the quantisation.
template <int IN, int PS>
__global__ void __launch_bounds__(kAppThreads)
k_paged_append(const QkvRows x, int Hq, int Hkv, const PageView pv,
               const __grid_constant__ RopeTurns rope, const int32_t *__restrict__ seq,
               const int32_t *__restrict__ pos, bf16 *__restrict__ q, uint8_t *__restrict__ kp,
               uint8_t *__restrict__ vp, float *__restrict__ ks, float *__restrict__ vs, int n_qb,
               int rpb, int slots, unsigned *err) {
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    constexpr int H2 = kPagedDh / 2, R = PS / kAppHalves;
    const int T = x.T, tid = threadIdx.x, lane = tid & 31;
    const int hw = tid / 16, i = 4 * (tid % 16);
    __shared__ __align__(16) float sn_s[kAppQTokens][H2], cs_s[kAppQTokens][H2];
    __shared__ int in_s[kAppQTokens];
    __shared__ int tok_at[PS];
    __shared__ uint32_t starts[kAppGroup / 32];
    __shared__ float red[kAppHalves], ratio_s[kAppRows];
    int b = (int)blockIdx.x;
    if (b < n_qb) {
        const int nrb = (Hq + kAppHalves - 1) / kAppHalves;
        const int t0 = b / nrb * kAppQTokens, hr = b % nrb * kAppHalves + hw;
        const int nt = min(kAppQTokens, T - t0);
        float av[kAppQTokens][4], bv[kAppQTokens][4];
#pragma unroll
        for (int u = 0; u < kAppQTokens; ++u)
            if (hr < Hq && u < nt) load_pairs<IN>(x, t0 + u, hr, i, av[u], bv[u]);
        static_assert(kAppQTokens * H2 == kAppThreads, "an angle a thread");
        if (tid / H2 < nt) {
            const int t = t0 + tid / H2, sq = seq[t], p = pos[t];
            const bool in = pv.inside(sq, p);
            rope_sincos(rope.r[tid % H2], in ? p : 0, sn_s[tid / H2][tid % H2],
                        cs_s[tid / H2][tid % H2]);
            if (tid % H2 == 0) {
                in_s[tid / H2] = in;
                // (seq < 0: a padding token, no error)
                if (!in && sq >= 0 && b % nrb == 0) set_error(err, kErrIndex);
            }
        }
        __syncthreads();
        if (hr >= Hq) return;
#pragma unroll
        for (int u = 0; u < kAppQTokens; ++u) {
            if (u >= nt) break;
            const float4 sn = *reinterpret_cast<const float4 *>(&sn_s[u][i]);
            const float4 cs = *reinterpret_cast<const float4 *>(&cs_s[u][i]);
            turn(av[u][0], bv[u][0], sn.x, cs.x);
            turn(av[u][1], bv[u][1], sn.y, cs.y);
            turn(av[u][2], bv[u][2], sn.z, cs.z);
            turn(av[u][3], bv[u][3], sn.w, cs.w);
            const bool in = in_s[u];  // else a row of zeros
            bf16 *o = q + ((size_t)(t0 + u) * Hq + hr) * kPagedDh + i;
            __nv_bfloat162 w[4] = {
                __floats2bfloat162_rn(av[u][0], av[u][1]), __floats2bfloat162_rn(av[u][2], av[u][3]),
                __floats2bfloat162_rn(bv[u][0], bv[u][1]), __floats2bfloat162_rn(bv[u][2], bv[u][3])};
            const uint32_t *w4 = reinterpret_cast<const uint32_t *>(w);
            *reinterpret_cast<uint2 *>(o) = in ? make_uint2(w4[0], w4[1]) : make_uint2(0u, 0u);
            *reinterpret_cast<uint2 *>(o + H2) = in ? make_uint2(w4[2], w4[3]) : make_uint2(0u, 0u);
        }
        return;
    }
    b -= n_qb;
    const int nrb = (2 * Hkv + rpb - 1) / rpb;
    const int slot = b % slots, rb = b / slots % nrb, g0 = b / slots / nrb * kAppGroup;
    const int r_end = min((rb + 1) * rpb, 2 * Hkv);
    if (tid < kAppGroup) {
        const int t = g0 + tid;
        bool start = false;
        if (t < T) {
            const int sq = seq[t], p = pos[t];
            start = pv.inside(sq, p) &&
                    !(t > 0 && (p & (PS - 1)) != 0 && seq[t - 1] == sq && pos[t - 1] == p - 1);
        }
        const uint32_t m = __ballot_sync(0xffffffffu, start);
        if (lane == 0) starts[tid / 32] = m;
    }
    if (tid < PS) tok_at[tid] = -1;
    __syncthreads();
    uint32_t words[kAppGroup / 32];
    int n_starts = 0;
#pragma unroll
    for (int w = 0; w < kAppGroup / 32; ++w) {
        words[w] = starts[w];
        n_starts += __popc(words[w]);
    }
#pragma unroll 1
    for (int s = slot; s < n_starts; s += slots) {
        const int t = g0 + nth_bit(words, s);
        const int sq = seq[t], p0 = pos[t], pi = p0 / PS;
        const int pg = pv.page(sq, pi);
        if (s != slot) {  // (the rows of the start before are done with tok_at)
            __syncthreads();
            if (tid < PS) tok_at[tid] = -1;
            __syncthreads();
        }
        bool earlier = false;
        auto seen = [&](int j, int sj, int pj) {
            if (j >= T || sj != sq || pj < 0 || pj / PS != pi) return;
            earlier |= j < t;
            atomicMax(&tok_at[pj & (PS - 1)], j);
        };
        // (four of them a load; the last may lie past the call's, not past the
        // arrays' 16-byte units)
        const int n4 = T / 4;
#pragma unroll 4
        for (int j = tid; j < n4; j += kAppThreads) {
            const int4 s4 = __ldg(reinterpret_cast<const int4 *>(seq) + j);
            const int4 p4 = __ldg(reinterpret_cast<const int4 *>(pos) + j);
            seen(4 * j, s4.x, p4.x);
            seen(4 * j + 1, s4.y, p4.y);
            seen(4 * j + 2, s4.z, p4.z);
            seen(4 * j + 3, s4.w, p4.w);
        }
        if (tid < T - 4 * n4) seen(4 * n4 + tid, seq[4 * n4 + tid], pos[4 * n4 + tid]);
        if (__syncthreads_or(earlier)) continue;  // another start leads this page
        const int n_in = __syncthreads_count(tid < PS && tok_at[tid] >= 0);
        if (pg < 0) {
            if (rb == 0 && tid == 0) set_error(err, kErrIndex);
            continue;
        }
        const bool fresh = tok_at[0] >= 0;
        // key or value row hr of the page: its scale, its numbers
        auto scale_at = [&](int hr) {
            return (hr < Hkv ? ks : vs) + (size_t)pg * Hkv + (hr < Hkv ? hr : hr - Hkv);
        };
        auto rows_at = [&](int hr) {
            return (hr < Hkv ? kp : vp) +
                   ((size_t)pg * Hkv + (hr < Hkv ? hr : hr - Hkv)) * PS * kPagedDh;
        };
        auto magnitude = [&](const float (&a)[4], const float (&c)[4], float mx) {
#pragma unroll
            for (int e = 0; e < 4; ++e) mx = fmaxf(mx, fmaxf(finite_abs(a[e]), finite_abs(c[e])));
            return mx;
        };
        auto half_max = [&](float mx) {
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            return mx;
        };
        auto turn_key = [&](float (&a)[4], float (&c)[4], int p) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float sn, cs;
                rope_sincos(rope.r[i + e], p, sn, cs);
                turn(a[e], c[e], sn, cs);
            }
        };
        if (n_in == 1) {
            const int hr = rb * rpb + hw;  // (rpb is at most the halves)
            const bool mine = hr < r_end;
            float a[4] = {0.f, 0.f, 0.f, 0.f}, c[4] = {0.f, 0.f, 0.f, 0.f}, old = 1.f;
            if (mine) {
                load_pairs<IN>(x, t, Hq + hr, i, a, c);
                old = *scale_at(hr);
                if (hr < Hkv) turn_key(a, c, p0);
            }
            const float need = scale_for(half_max(magnitude(a, c, 0.f)));
            const float scale = fresh ? need : fmaxf(old, need);
            const bool grown = mine && !fresh && scale != old;
            if (mine) {
                uint8_t *row = rows_at(hr) + (size_t)(p0 & (PS - 1)) * kPagedDh + i;
                *reinterpret_cast<uint32_t *>(row) = quantise(a, scale);
                *reinterpret_cast<uint32_t *>(row + H2) = quantise(c, scale);
                if (i == 0) {
                    *scale_at(hr) = scale;
                    ratio_s[hw] = grown ? old / scale : 1.f;
                }
            }
            if (!__syncthreads_or(grown)) continue;
            // the other rows of the pages that grew, by the whole block
            for (int r = 0; r < r_end - rb * rpb; ++r) {
                const float ratio = ratio_s[r];
                if (ratio == 1.f) continue;
                uint8_t *rows = rows_at(rb * rpb + r);
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    const int o = hw + k * kAppHalves;
                    if (o == (p0 & (PS - 1))) continue;
                    uint2 *p8 = reinterpret_cast<uint2 *>(rows + (size_t)o * kPagedDh + 2 * i);
                    uint2 v = *p8;
                    v.x = rescale(v.x, ratio);
                    v.y = rescale(v.y, ratio);
                    *p8 = v;
                }
            }
            continue;
        }
        int tok[R];
#pragma unroll
        for (int k = 0; k < R; ++k) tok[k] = tok_at[hw + k * kAppHalves];
#pragma unroll 1
        for (int hr = rb * rpb; hr < r_end; ++hr) {
            uint8_t *rows = rows_at(hr);
            const float old = *scale_at(hr);
            float a[R][4], c[R][4];
            float mx = 0.f;
#pragma unroll
            for (int k = 0; k < R; ++k) {
#pragma unroll
                for (int e = 0; e < 4; ++e) a[k][e] = c[k][e] = 0.f;
                if (tok[k] >= 0) load_pairs<IN>(x, tok[k], Hq + hr, i, a[k], c[k]);
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (tok[k] < 0) continue;
                if (hr < Hkv) turn_key(a[k], c[k], pi * PS + hw + k * kAppHalves);
                mx = magnitude(a[k], c[k], mx);
            }
            mx = half_max(mx);
            if (i == 0) red[hw] = mx;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kAppHalves; ++u) mx = fmaxf(mx, red[u]);
            __syncthreads();
            const float need = scale_for(mx);
            const float scale = fresh ? need : fmaxf(old, need);
            if (tid == 0) *scale_at(hr) = scale;
            const bool grown = !fresh && scale != old;
            const float ratio = old / scale;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                uint8_t *row = rows + (size_t)(hw + k * kAppHalves) * kPagedDh;
                if (tok[k] >= 0) {
                    *reinterpret_cast<uint32_t *>(row + i) = quantise(a[k], scale);
                    *reinterpret_cast<uint32_t *>(row + H2 + i) = quantise(c[k], scale);
                } else if (grown) {
                    uint2 *p8 = reinterpret_cast<uint2 *>(row + 2 * i);
                    uint2 v = *p8;
                    v.x = rescale(v.x, ratio);
                    v.y = rescale(v.y, ratio);
                    *p8 = v;
                }
            }
        }
    }
}

template <int IN>
const void *append_kernel(int ps) {
    switch (ps) {
        case 16: return (const void *)k_paged_append<IN, 16>;
        case 32: return (const void *)k_paged_append<IN, 32>;
        case 64: return (const void *)k_paged_append<IN, 64>;
        default: return (const void *)k_paged_append<IN, 128>;
    }
}

cudaError_t launch_append(const QkvRows &rows, int in, const moe_sa_dims &d,
                          const moe_paged_dims &pd, const int32_t *seq, const int32_t *pos,
                          const int32_t *table, void *q, void *kp, void *vp, float *ks, float *vs,
                          cudaStream_t st) {
    int Hq = d.n_heads, Hkv = d.n_kv_heads;
    const int T = rows.T;
    QkvRows x = rows;
    PageView pv{table, pd.n_seq, pd.max_pages, pd.n_pages, 31 - __builtin_clz(pd.page_size)};
    RopeTurns rope = rope_turns(d.rope_base);
    bf16 *qp = static_cast<bf16 *>(q);
    uint8_t *k8 = static_cast<uint8_t *>(kp), *v8 = static_cast<uint8_t *>(vp);
    unsigned *err = device_info().err;
    int n_qb = (Hq + kAppHalves - 1) / kAppHalves * ((T + kAppQTokens - 1) / kAppQTokens);
    // a decode batch: all rows of a token in one block; larger calls, which have
    // more pages with many tokens: few rows, the look through the call shared by
    // four of them where it is long
    int rpb = T <= kAppGroup ? kAppRows : T <= 1024 ? 2 : 4;
    int slots = T <= kAppGroup ? T : T <= 1024 ? 32 : 8;
    const int groups = (T + kAppGroup - 1) / kAppGroup;
    const int n_kb = groups * ((2 * Hkv + rpb - 1) / rpb) * slots;
    const void *kern = in == kInBf16  ? append_kernel<kInBf16>(pd.page_size)
                       : in == kInF32 ? append_kernel<kInF32>(pd.page_size)
                                      : append_kernel<kInParts>(pd.page_size);
    void *args[] = {&x,  &Hq, &Hkv, &pv, &rope, &seq, &pos,   &qp,
                    &k8, &v8, &ks,  &vs, &n_qb, &rpb, &slots, &err};
    LaunchScope ls("paged_append", st);
    return launch_pdl(kern, dim3((unsigned)(n_qb + n_kb)), dim3(kAppThreads), 0, st, args);
}

// The tokens that are attended one by one (in their order), the position tiles
// ahead of each, and the decode attention's counters at zero.  One block.
constexpr int kPlanThreads = 1024;

__global__ void __launch_bounds__(kPlanThreads)
k_paged_plan(int T, const PageView pv, const int32_t *__restrict__ seq,
             const int32_t *__restrict__ pos, const PagedList l, const PlanArgs pa) {
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    __shared__ long long sums[kPlanThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < kPagedMaxCtas; i += kPlanThreads) l.count[i] = 0;
    int n = T;
    if (pa.plan.head) {  // only those that no tile holds
        plan_attention<kPlanThreads>(T, pa);
        __syncthreads();
        n = pa.plan.head->n_left;
    }
    long long run = 0;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + tid;
        int nt = 0;
        if (i < n) {
            const int t = pa.plan.head ? pa.plan.left[i] : i, p = pos[t];
            if (!pa.plan.head) l.list[i] = t;
            nt = pv.inside(seq[t], p) ? p / kPagedTile + 1 : 1;
        }
        long long v = nt;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        if (lane == 31) sums[warp] = v;
        __syncthreads();
        if (warp == 0) {
            long long s = sums[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long u = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= o) s += u;
            }
            sums[lane] = s;
        }
        __syncthreads();
        const long long ahead = run + (warp > 0 ? sums[warp - 1] : 0) + v - nt;
        if (i < n) l.before[i] = ahead;
        run += sums[kPlanThreads / 32 - 1];
        __syncthreads();
    }
    if (tid == 0) {
        l.before[n] = run;
        *l.n_list = n;
    }
}

// ---- host ------------------------------------------------------------------------

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool ok_ptr(const void *p) { return p != nullptr && aligned16(p); }
moe_status cuda_status(cudaError_t e) { return e == cudaSuccess ? MOE_OK : MOE_ERR_CUDA; }

// Workspace of moe_paged_attend.
struct PagedWs {
    size_t n_list, count, list, before, head, tiles, part, total;
};

PagedWs paged_ws(int64_t T) {
    auto up = [](size_t v) { return (v + 255) & ~size_t(255); };
    PagedWs L{};
    size_t o = 0;
    L.n_list = o; o += up(4);
    L.count = o; o += up(kPagedMaxCtas * 4);
    L.list = o; o += up((size_t)T * 4);
    L.before = o; o += up(((size_t)T + 1) * 8);
    L.head = o; o += up(sizeof(AttnPlanHead));
    L.tiles = o; o += up((size_t)(T / kAttnTileMinRows) * sizeof(int4));
    L.part = o; o += up(kPagedPartFloats * 4);
    L.total = o;
    return L;
}

template <typename P>
P *at(void *ws, size_t off) {
    return reinterpret_cast<P *>(static_cast<char *>(ws) + off);
}

// Whether a call's tokens are sorted into tiles and the rest (as in attn.cu).
constexpr int kPagedPlanTokens = 48;  // beyond one for each sequence
bool planned(int T, int n_seq) { return T >= kAttnTile || T - n_seq >= kPagedPlanTokens; }

cudaError_t attend(const PagedAttn &a, void *ws, cudaStream_t st) {
    const PagedWs L = paged_ws(a.T);
    PagedList l{at<int>(ws, L.n_list), at<int>(ws, L.list), at<long long>(ws, L.before),
                at<int>(ws, L.count)};
    PlanArgs pa{a.seq, a.pos, a.pv.n_seq, a.pv.max_pages << a.pv.shift, {}};
    if (planned(a.T, a.pv.n_seq))
        pa.plan = AttnPlan{at<AttnPlanHead>(ws, L.head), at<int4>(ws, L.tiles), l.list};
    {
        int T = a.T;
        PageView pv = a.pv;
        const int32_t *seq = a.seq, *pos = a.pos;
        void *args[] = {&T, &pv, &seq, &pos, &l, &pa};
        LaunchScope ls("paged_plan", st);
        cudaError_t e =
            launch_pdl((const void *)k_paged_plan, dim3(1), dim3(kPlanThreads), 0, st, args);
        if (e != cudaSuccess) return e;
    }
    if (pa.plan.head) {
        cudaError_t e = launch_paged_prefill_tc(a, pa.plan, st);
        if (e != cudaSuccess) return e;
    }
    return launch_paged_decode_tc(a, l, at<float>(ws, L.part), st);
}

moe_status check_paged(const moe_sa_dims *d, const moe_paged_dims *pd) {
    size_t n = 0;
    moe_status s = moe_sa_workspace_size(d, 0, &n);  // the shape's own limits
    if (s != MOE_OK) return s;
    if (!pd) return MOE_ERR_INVALID_ARG;
    if (pd->n_pages < 1 || pd->n_seq < 1 || pd->max_pages < 1 || pd->page_size < 1)
        return MOE_ERR_INVALID_ARG;
    if (pd->page_size != 16 && pd->page_size != 32 && pd->page_size != 64 && pd->page_size != 128)
        return MOE_ERR_UNSUPPORTED;
    const int64_t most = (1LL << 31) - 1;
    if ((int64_t)pd->n_pages * d->n_kv_heads * pd->page_size > most ||
        (int64_t)pd->max_pages * pd->page_size > most)
        return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

moe_status check_paged_call(const moe_sa_dims *d, const moe_paged_dims *pd, int32_t T,
                            const int32_t *seq, const int32_t *pos, const int32_t *table,
                            const void *kp, const void *vp, const float *ks, const float *vs) {
    moe_status s = check_paged(d, pd);
    if (s != MOE_OK) return s;
    if (T < 0 || T > kPagedMaxTokens) return MOE_ERR_INVALID_ARG;
    if (T > 0 && (!ok_ptr(seq) || !ok_ptr(pos) || !ok_ptr(table) || !ok_ptr(kp) || !ok_ptr(vp) ||
                  !ok_ptr(ks) || !ok_ptr(vs)))
        return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

moe_status moe_paged_workspace_size(const moe_sa_dims *dims, int32_t max_tokens, size_t *bytes) {
    size_t n = 0;
    moe_status s = moe_sa_workspace_size(dims, 0, &n);
    if (s != MOE_OK) return s;
    if (!bytes || max_tokens < 0 || max_tokens > kPagedMaxTokens) return MOE_ERR_INVALID_ARG;
    *bytes = paged_ws(max_tokens).total;
    return MOE_OK;
}

moe_status moe_paged_append(const moe_sa_dims *dims, const moe_paged_dims *paged, int32_t T,
                            const void *qkv, int32_t qkv_dtype, const int32_t *seq,
                            const int32_t *pos, const int32_t *page_table, void *q, void *k_pages,
                            void *v_pages, float *k_scale, float *v_scale, moe_stream_t stream) {
    MOE_INJECT("moe_paged_append");
    moe_status s = check_paged_call(dims, paged, T, seq, pos, page_table, k_pages, v_pages,
                                    k_scale, v_scale);
    if (s != MOE_OK) return s;
    if (qkv_dtype != MOE_F32 && qkv_dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!ok_ptr(qkv) || !ok_ptr(q)) return MOE_ERR_INVALID_ARG;
    const QkvRows rows{qkv, (dims->n_heads + 2 * dims->n_kv_heads) * kPagedDh, T, 1, 0, {}};
    return cuda_status(launch_append(rows, qkv_dtype == MOE_BF16 ? kInBf16 : kInF32, *dims, *paged,
                                     seq, pos, page_table, q, k_pages, v_pages, k_scale, v_scale,
                                     (cudaStream_t)stream));
}

moe_status moe_paged_attend(const moe_sa_dims *dims, const moe_paged_dims *paged, int32_t T,
                            const void *q, const int32_t *seq, const int32_t *pos,
                            const int32_t *page_table, const void *k_pages, const void *v_pages,
                            const float *k_scale, const float *v_scale, void *ctx, void *ws,
                            size_t ws_bytes, moe_stream_t stream) {
    MOE_INJECT("moe_paged_attend");
    moe_status s = check_paged_call(dims, paged, T, seq, pos, page_table, k_pages, v_pages,
                                    k_scale, v_scale);
    if (s != MOE_OK) return s;
    if (T == 0) return MOE_OK;
    if (!ok_ptr(q) || !ok_ptr(ctx)) return MOE_ERR_INVALID_ARG;
    size_t need = 0;
    if ((s = moe_paged_workspace_size(dims, T, &need)) != MOE_OK) return s;
    if (!ok_ptr(ws) || ws_bytes < need) return MOE_ERR_WORKSPACE;
    const PagedAttn a{T,
                      dims->n_heads,
                      dims->n_kv_heads,
                      paged->page_size,
                      PageView{page_table, paged->n_seq, paged->max_pages, paged->n_pages,
                               31 - __builtin_clz(paged->page_size)},
                      seq,
                      pos,
                      q,
                      k_pages,
                      v_pages,
                      k_scale,
                      v_scale,
                      ctx};
    return cuda_status(attend(a, ws, (cudaStream_t)stream));
}

}  // extern "C"
