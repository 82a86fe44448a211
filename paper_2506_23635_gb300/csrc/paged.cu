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
// the SMs do little).  r_i comes from a power and a division of 53 bits, to 2^-54.6 of
// a turn (base 500000: 2^-55.5), so the angle is off by p times that, by 2^-32 where
// the product is cut to 32 bits and by 2^-26 where those become fp32: below 2^-24 of
// a turn (2^-21.4 in radians) at the last position of all, 2^30.
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

constexpr int kAppThreads = 512;
constexpr int kAppHalves = kAppThreads / 16;  // half a warp takes a row, four pairs a lane
constexpr int kAppQTokens = 8;                // tokens of a block of the queries' part,
constexpr int kAppQRows = 16;                 // and head rows: a row of four of them a half
constexpr int kAppQEach = kAppQTokens * kAppQRows / kAppHalves;
constexpr int kAppMaxGroup = 128;  // tokens whose pages a block looks after, at most

// The pair's rotation.
__device__ __forceinline__ void turn(float &a, float &b, float sn, float cs) {
    const float u = a, v = b;
    a = u * cs - v * sn;
    b = v * cs + u * sn;
}

// A result y that was cut off, its last bit set where something was: rounded to a
// few bits it gives what the exact result does (after a rounding to nearest it may
// not).
__device__ __forceinline__ float sticky(float y, bool inexact) {
    return inexact ? __uint_as_float(__float_as_uint(y) | 1u) : y;
}

// All scales that this kernel gives are powers of two, division by which is exact as
// a product; a caller's own cache may hold others, by which numbers are divided (q
// the quotient cut off; x - q scale is exact; NaN and infinities give NaN).
__device__ __forceinline__ bool power_of_two(float scale) {
    return (__float_as_uint(scale) & 0x7fffffu) == 0;
}
__device__ __forceinline__ void divide(float (&x)[4], float scale) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float q = __fdiv_rz(x[e], scale);
        x[e] = sticky(q, fmaf(-q, scale, x[e]) != 0.f);
    }
}

// Four numbers x inv, as they are stored.
__device__ __forceinline__ uint32_t quantise(const float (&x)[4], float inv) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = storable(x[e]) * inv;
    return e4m3x2(y[0], y[1]) | e4m3x2(y[2], y[3]) << 16;
}

// The multiplier of a page's other rows; negative where they were zeros, NaN
// among them, under a scale of zero.
__device__ __forceinline__ float growth(float old, float scale) {
    return old == 0.f ? -1.f : old / scale;
}

// Four stored numbers times ratio, rounded again, once.
__device__ __forceinline__ float times(float x, float ratio) {
    const float y = __fmul_rz(x, ratio);
    return sticky(y, fmaf(x, ratio, -y) != 0.f);
}
__device__ __forceinline__ uint32_t rescale(uint32_t v, float ratio) {
    if (ratio < 0.f) return 0u;
    const float2 f0 = e4m3x2_to_float2(v & 0xffffu), f1 = e4m3x2_to_float2(v >> 16);
    return e4m3x2(times(f0.x, ratio), times(f0.y, ratio)) |
           e4m3x2(times(f1.x, ratio), times(f1.y, ratio)) << 16;
}

// Blocks [0, n_kb): keys and values, each a row (key or value head) of the pages
// that a group of gs consecutive tokens starts.  The tokens of a call that lie in
// one page are found from the first of them: a token leads its page if no earlier
// token of the call lies there.  Only one that does not follow its
// predecessor inside the page can (a start); the block compares the whole call's
// tokens, which may come in any order, with the group's starts.  Pages with one
// token (decode): half a warp each, all side by side; the others one after the
// other, the page's tokens in registers between their maximum and the
// quantisation.  The blocks after them: queries, kAppQRows head rows of
// kAppQTokens tokens, half a warp a row of four of them.
//
// Bound: the chain of dependent loads of a start, its page and its row (48 + 2 x 8
// heads: one token 3.9 us, 61 tokens 6.1, 529 tokens 9.2), and where there are many
// tokens that chain over the two blocks that an SM holds beside the queries' bytes
// (12,000 tokens 87.5 us, 4.2 TB/s; the queries' part alone 56, 5.2 TB/s).
// MANY: a block takes `per` rows of its group, else one.
template <int IN, int PS, bool MANY>
__global__ void __launch_bounds__(kAppThreads, 2)
k_paged_append(const QkvRows x, int Hq, int Hkv, const PageView pv,
               const __grid_constant__ RopeTurns rope, const int32_t *__restrict__ seq,
               const int32_t *__restrict__ pos, bf16 *__restrict__ q, uint8_t *__restrict__ kp,
               uint8_t *__restrict__ vp, float *__restrict__ ks, float *__restrict__ vs, int n_kb,
               int gs, int per, unsigned *err) {
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    constexpr int H2 = kPagedDh / 2, R = (PS + kAppHalves - 1) / kAppHalves;
    const int T = x.T, tid = threadIdx.x, lane = tid & 31;
    const int hw = tid / 16, i = 4 * (tid % 16);
    if ((int)blockIdx.x >= n_kb) {
        __shared__ __align__(16) float sn_s[kAppQTokens][H2], cs_s[kAppQTokens][H2];
        __shared__ int in_s[kAppQTokens];
        const int b = (int)blockIdx.x - n_kb;
        const int nrb = (Hq + kAppQRows - 1) / kAppQRows;
        const int t0 = b / nrb * kAppQTokens, hr = b % nrb * kAppQRows + hw % kAppQRows;
        const int nt = min(kAppQTokens, T - t0), u0 = hw / kAppQRows * kAppQEach;
        float av[kAppQEach][4], bv[kAppQEach][4];
#pragma unroll
        for (int u = 0; u < kAppQEach; ++u)
            if (hr < Hq && u0 + u < nt) load_pairs<IN>(x, t0 + u0 + u, hr, i, av[u], bv[u]);
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
        for (int u = 0; u < kAppQEach; ++u) {
            if (u0 + u >= nt) break;
            const float4 sn = *reinterpret_cast<const float4 *>(&sn_s[u0 + u][i]);
            const float4 cs = *reinterpret_cast<const float4 *>(&cs_s[u0 + u][i]);
            turn(av[u][0], bv[u][0], sn.x, cs.x);
            turn(av[u][1], bv[u][1], sn.y, cs.y);
            turn(av[u][2], bv[u][2], sn.z, cs.z);
            turn(av[u][3], bv[u][3], sn.w, cs.w);
            const bool in = in_s[u0 + u];  // else a row of zeros
            bf16 *o = q + ((size_t)(t0 + u0 + u) * Hq + hr) * kPagedDh + i;
            __nv_bfloat162 w[4] = {
                __floats2bfloat162_rn(av[u][0], av[u][1]), __floats2bfloat162_rn(av[u][2], av[u][3]),
                __floats2bfloat162_rn(bv[u][0], bv[u][1]), __floats2bfloat162_rn(bv[u][2], bv[u][3])};
            const uint32_t *w4 = reinterpret_cast<const uint32_t *>(w);
            *reinterpret_cast<uint2 *>(o) = in ? make_uint2(w4[0], w4[1]) : make_uint2(0u, 0u);
            *reinterpret_cast<uint2 *>(o + H2) = in ? make_uint2(w4[2], w4[3]) : make_uint2(0u, 0u);
        }
        return;
    }
    __shared__ int n_s, n_grown;
    __shared__ int t_s[kAppMaxGroup], page_s[kAppMaxGroup], count_s[kAppMaxGroup];
    __shared__ int2 at_s[kAppMaxGroup];      // a start's sequence, page index
    __shared__ int grown_s[kAppMaxGroup];    // starts whose page's scale grew
    __shared__ float ratio_s[kAppMaxGroup];  // and by what
    constexpr int kFew = 2;  // starts whose pages' tokens are found in one look
    __shared__ int tok_at[kFew][PS];
    __shared__ float red[kAppHalves];
    if constexpr (!MANY) per = 1;
    const int n_hr = 2 * Hkv / per;  // blocks of a group
    const int hr0 = (int)blockIdx.x % n_hr * per, g0 = (int)blockIdx.x / n_hr * gs;
    // a lane's pairs' rates (read from the parameters by 16 different addresses a
    // half warp, so once)
    uint64_t rate[4] = {0, 0, 0, 0};
    if (hr0 < Hkv) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            rate[e] = rope.r[i + e];
            asm volatile("" : "+l"(rate[e]));
        }
    }
    if (tid == 0) n_s = n_grown = 0;
    for (int o = tid; o < kFew * PS; o += kAppThreads) (&tok_at[0][0])[o] = -1;
    __syncthreads();
    if (tid < gs && g0 + tid < T) {
        const int t = g0 + tid, sq = seq[t], p = pos[t];
        if (pv.inside(sq, p) &&
            !(t > 0 && (p & (PS - 1)) != 0 && seq[t - 1] == sq && pos[t - 1] == p - 1)) {
            const int s = atomicAdd(&n_s, 1);  // (in any order: nothing depends on it)
            t_s[s] = t;
            at_s[s] = make_int2(sq, p / PS);
            count_s[s] = 0;
            const int pg = pv.page(sq, p / PS);
            page_s[s] = pg;
            if (pg < 0 && hr0 == 0) set_error(err, kErrIndex);
        }
    }
    __syncthreads();
    const int n_starts = n_s;
    if (n_starts == 0) return;
    // how many tokens of the call lie in each start's page; where an earlier one
    // does, that one leads the page and this start has none
    const int n4 = T / 4;
    if (n_starts <= kFew) {  // a thread a token, and the page's tokens right away
        int2 at[kFew];  // sequence, first position of the page
#pragma unroll
        for (int s = 0; s < kFew; ++s) {
            at[s] = at_s[min(s, n_starts - 1)];
            at[s].y *= PS;
        }
        // zero where the token lies in a start's page: two operations a start (whole
        // comparisons: 12,000 tokens 95 us, 92.5 so)
        auto off = [&](int sq, int p) {
            unsigned m = 0xffffffffu;
#pragma unroll
            for (int s = 0; s < kFew; ++s)
                m = min(m, (unsigned)((sq ^ at[s].x) | ((p ^ at[s].y) & ~(PS - 1))));
            return m;
        };
        auto compare = [&](int t, int sq, int p) {
            if (off(sq, p) != 0u) return;
            for (int s = 0; s < n_starts; ++s) {
                if (at_s[s].x != sq || at_s[s].y != p / PS) continue;
                if (t < t_s[s]) page_s[s] = -1;
                atomicAdd(&count_s[s], 1);
                atomicMax(&tok_at[s][p & (PS - 1)], t);
            }
        };
#pragma unroll 2
        for (int j = tid; j < n4; j += kAppThreads) {
            const int4 s4 = __ldg(reinterpret_cast<const int4 *>(seq) + j);
            const int4 p4 = __ldg(reinterpret_cast<const int4 *>(pos) + j);
            if (min(min(off(s4.x, p4.x), off(s4.y, p4.y)), min(off(s4.z, p4.z), off(s4.w, p4.w))) != 0u)
                continue;
            compare(4 * j, s4.x, p4.x);
            compare(4 * j + 1, s4.y, p4.y);
            compare(4 * j + 2, s4.z, p4.z);
            compare(4 * j + 3, s4.w, p4.w);
        }
        if (tid < T - 4 * n4) compare(4 * n4 + tid, seq[4 * n4 + tid], pos[4 * n4 + tid]);
    } else {  // a lane a start, a warp 32 tokens
        for (int s0 = 0; s0 < n_starts; s0 += 32) {
            const int s = s0 + lane;
            const int2 at = s < n_starts ? at_s[s] : make_int2(-1, -1);
            const int mine = s < n_starts ? t_s[s] : 0;
            int n = 0;
            bool early = false;
            for (int j0 = tid - lane; j0 < T; j0 += kAppThreads) {
                const int t = j0 + lane;
                const int sq = t < T ? seq[t] : -2, pi = t < T ? pos[t] >> pv.shift : -2;
#pragma unroll 8
                for (int u = 0; u < 32; ++u) {
                    // (every lane takes part in both)
                    const int su = __shfl_sync(0xffffffffu, sq, u);
                    const int pu = __shfl_sync(0xffffffffu, pi, u);
                    const bool here = su == at.x && pu == at.y;
                    n += here;
                    early |= here && j0 + u < mine;
                }
            }
            if (s < n_starts && n) atomicAdd(&count_s[s], n);
            if (s < n_starts && early) page_s[s] = -1;
        }
    }
    __syncthreads();
    // the largest magnitude; infinities are left out where there are any
    auto magnitude = [&](const float (&a)[4], const float (&c)[4], float mx, bool all) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            mx = all ? fmaxf(mx, fmaxf(fabsf(a[e]), fabsf(c[e])))
                     : fmaxf(mx, fmaxf(finite_abs(a[e]), finite_abs(c[e])));
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
            rope_sincos(rate[e], p, sn, cs);
            turn(a[e], c[e], sn, cs);
        }
    };
#pragma unroll 1
    for (int hr = hr0; hr < hr0 + per; ++hr) {
        const bool key = hr < Hkv;
        const int h = key ? hr : hr - Hkv;
        float *scales = (key ? ks : vs) + h;
        uint8_t *pool = (key ? kp : vp) + (size_t)h * PS * kPagedDh;
        auto rows_of = [&](int pg) { return pool + (size_t)pg * Hkv * PS * kPagedDh; };
        if (MANY && hr != hr0) {
            __syncthreads();  // (all have read the last row's)
            if (tid == 0) n_grown = 0;
            __syncthreads();
        }
        // pages with one token of the call
#pragma unroll 1
        for (int s0 = 0; s0 < n_starts; s0 += kAppHalves) {
            const int s = s0 + hw;
            if (!__any_sync(0xffffffffu, s < n_starts && count_s[s] == 1)) continue;
            const bool mine = s < n_starts && count_s[s] == 1 && page_s[s] >= 0;
            float a[4] = {0.f, 0.f, 0.f, 0.f}, c[4] = {0.f, 0.f, 0.f, 0.f}, old = 1.f;
            int p = 0, pg = 0;
            if (mine) {
                const int t = t_s[s];
                pg = page_s[s];
                load_pairs<IN>(x, t, Hq + hr, i, a, c);
                old = scales[(size_t)pg * Hkv];
                p = pos[t];
                if (key) turn_key(a, c, p);
            }
            float mx = half_max(magnitude(a, c, 0.f, true));
            if (__any_sync(0xffffffffu, mx == INFINITY)) mx = half_max(magnitude(a, c, 0.f, false));
            const float need = scale_for(mx);
            if (!mine) continue;
            const bool fresh = (p & (PS - 1)) == 0;
            const float scale = fresh ? need : fmaxf(old, need);
            uint8_t *row = rows_of(pg) + (size_t)(p & (PS - 1)) * kPagedDh + i;
            float inv = 1.f / scale;
            if (!power_of_two(scale)) {
                divide(a, scale);
                divide(c, scale);
                inv = 1.f;
            }
            *reinterpret_cast<uint32_t *>(row) = quantise(a, inv);
            *reinterpret_cast<uint32_t *>(row + H2) = quantise(c, inv);
            if (i == 0) {
                scales[(size_t)pg * Hkv] = scale;
                if (!fresh && scale != old) {
                    const int n = atomicAdd(&n_grown, 1);
                    grown_s[n] = s;
                    ratio_s[n] = growth(old, scale);
                }
            }
        }
        __syncthreads();
        // the other rows of those whose scale grew, by the whole block
#pragma unroll 1
        for (int r = hw; r < n_grown * PS; r += 4 * kAppHalves) {
            uint2 v[4];
            uint2 *p8[4];
            float ratio[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int rr = r + u * kAppHalves, n = rr / PS, o = rr % PS;
                p8[u] = nullptr;
                if (n >= n_grown) continue;
                const int s = grown_s[n];
                if (o == (pos[t_s[s]] & (PS - 1))) continue;
                ratio[u] = ratio_s[n];
                p8[u] = reinterpret_cast<uint2 *>(rows_of(page_s[s]) + (size_t)o * kPagedDh + 2 * i);
                v[u] = *p8[u];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (p8[u]) *p8[u] = make_uint2(rescale(v[u].x, ratio[u]), rescale(v[u].y, ratio[u]));
        }
        // the others
#pragma unroll 1
        for (int s = 0; s < n_starts; ++s) {
            if (count_s[s] <= 1 || page_s[s] < 0) continue;
            const int pg = page_s[s], sq = at_s[s].x, pi = at_s[s].y;
            int *toks = tok_at[n_starts <= kFew ? s : 0];
            if (n_starts > kFew) {
                __syncthreads();
                if (tid < PS) toks[tid] = -1;
                __syncthreads();
                auto seen = [&](int t, int st, int p) {
                    if (st == sq && p >= 0 && p / PS == pi) atomicMax(&toks[p & (PS - 1)], t);
                };
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
                __syncthreads();
            }
            const bool fresh = toks[0] >= 0;
            int tok[R];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const int o = hw + k * kAppHalves;
                tok[k] = o < PS ? toks[o] : -1;
            }
            uint8_t *rows = rows_of(pg);
            const float old = scales[(size_t)pg * Hkv];
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
                if (key) turn_key(a[k], c[k], pi * PS + hw + k * kAppHalves);
                mx = magnitude(a[k], c[k], mx, true);
            }
            auto block_max = [&]() {
                mx = half_max(mx);
                if (i == 0) red[hw] = mx;
                __syncthreads();
#pragma unroll
                for (int u = 0; u < kAppHalves; ++u) mx = fmaxf(mx, red[u]);
            };
            block_max();
            if (mx == INFINITY) {  // (the same in every thread)
                __syncthreads();
                mx = 0.f;
#pragma unroll
                for (int k = 0; k < R; ++k) mx = magnitude(a[k], c[k], mx, false);
                block_max();
            }
            const float need = scale_for(mx);
            const float scale = fresh ? need : fmaxf(old, need);
            const bool grown = !fresh && scale != old;
            const float ratio = growth(old, scale);
            float inv = 1.f / scale;
            if (!power_of_two(scale)) {
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    divide(a[k], scale);
                    divide(c[k], scale);
                }
                inv = 1.f;
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                uint8_t *row = rows + (size_t)(hw + k * kAppHalves) * kPagedDh;
                if (tok[k] >= 0) {
                    *reinterpret_cast<uint32_t *>(row + i) = quantise(a[k], inv);
                    *reinterpret_cast<uint32_t *>(row + H2 + i) = quantise(c[k], inv);
                } else if (grown && hw + k * kAppHalves < PS) {
                    uint2 *p8 = reinterpret_cast<uint2 *>(row + 2 * i);
                    uint2 v = *p8;
                    v.x = rescale(v.x, ratio);
                    v.y = rescale(v.y, ratio);
                    *p8 = v;
                }
            }
            __syncthreads();  // (the old scale is read by all, and red)
            if (tid == 0) scales[(size_t)pg * Hkv] = scale;
        }
    }
}

template <int IN, bool MANY>
const void *append_kernel(int ps) {
    switch (ps) {
        case 16: return (const void *)k_paged_append<IN, 16, MANY>;
        case 32: return (const void *)k_paged_append<IN, 32, MANY>;
        case 64: return (const void *)k_paged_append<IN, 64, MANY>;
        default: return (const void *)k_paged_append<IN, 128, MANY>;
    }
}
template <bool MANY>
const void *append_kernel(int in, int ps) {
    return in == kInBf16  ? append_kernel<kInBf16, MANY>(ps)
           : in == kInF32 ? append_kernel<kInF32, MANY>(ps)
                          : append_kernel<kInParts, MANY>(ps);
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
    const int n_qb = (Hq + kAppQRows - 1) / kAppQRows * ((T + kAppQTokens - 1) / kAppQTokens);
    // small groups where the tokens may all be starts; a page's worth of tokens
    // holds one or two otherwise
    int gs = T <= kAppMaxGroup ? kAppHalves : std::max(kAppHalves, (int)pd.page_size);
    // several rows a block, up to four, where there are blocks enough, one for each SM:
    // what a block finds out of its pages is half of its time (12,000 tokens, pages of
    // 128: one row 92.5 us, four 87.2, eight 99; 2048 tokens, pages of 64: one row 18.1
    // us, two 16.4, four, 128 blocks, 19.6; 529 tokens: one row 9.2, two, 136 blocks,
    // 13.8)
    const int groups = (T + gs - 1) / gs;
    int per = 1;
    while (per < 4 && 2 * Hkv % (2 * per) == 0 &&
           (long long)groups * 2 * Hkv / (2 * per) >= device_info().sm_count)
        per *= 2;
    int n_kb = groups * (2 * Hkv / per);
    const void *kern = per > 1 ? append_kernel<true>(in, pd.page_size)
                               : append_kernel<false>(in, pd.page_size);
    void *args[] = {&x,  &Hq, &Hkv, &pv, &rope, &seq, &pos,   &qp,
                    &k8, &v8, &ks,  &vs, &n_kb, &gs,  &per,  &err};
    LaunchScope ls("paged_append", st);
    return launch_pdl(kern, dim3((unsigned)(n_qb + n_kb)), dim3(kAppThreads), 0, st, args);
}

// The tokens that are attended one by one (in their order), the position tiles
// ahead of each, and the attention's counters at zero; in a call that is not sorted
// the decode attention's counters only.  One block.
constexpr int kPlanThreads = 1024;

__global__ void __launch_bounds__(kPlanThreads)
k_paged_plan(int T, const PageView pv, const int32_t *__restrict__ seq,
             const int32_t *__restrict__ pos, const PagedList l, const PlanArgs pa,
             int *unit_count) {
    ptx::grid_dependency_wait();
    // (after the wait: ahead of it one token of 2048 positions takes 10.4 us, 9.8 so)
    ptx::launch_dependents();
    __shared__ long long sums[kPlanThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < 2 * kPagedMaxCtas; i += kPlanThreads) l.count[i] = 0;
    if (!pa.plan.head) return;
    if (tid == 0) *l.released = 0;
    for (int i = tid; i < 2 * kPagedUnitParts; i += kPlanThreads) unit_count[i] = 0;
    const int n = plan_attention<kPlanThreads, kPagedTileMinRows>(T, pa);
    __syncthreads();
    long long run = 0;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + tid;
        int nt = 0;
        if (i < n) {
            const int t = l.list[i], p = pos[t];  // (where the plan has put them)
            nt = pv.inside(seq[t], p) ? p / kPagedTile + 1 : 0;
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
    if (n > 0) __syncthreads();
    // (nothing listed: who reads that reads nothing else, and need not be made to
    // wait for what this block stores; a prompt of 1000 tokens 29.9 us, 29.7 so)
    if (tid == 0 && n > 0)
        asm volatile("st.release.gpu.global.s32 [%0], %1;" ::"l"(l.released), "r"(n + 1) : "memory");
    else if (tid == 0)
        asm volatile("st.relaxed.gpu.global.s32 [%0], 1;" ::"l"(l.released) : "memory");
}

// ---- host ------------------------------------------------------------------------

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool ok_ptr(const void *p) { return p != nullptr && aligned16(p); }
moe_status cuda_status(cudaError_t e) { return e == cudaSuccess ? MOE_OK : MOE_ERR_CUDA; }

// Whether a call's tokens are sorted into tiles and the rest: the plan and the
// prefill attention's start cost 6 us and more beside tokens taken one by one (32
// tokens at position 3000: 33.0 us sorted, 33.7 not, beside 24 others 52.8 and 44.0).
// The table's rows are all that the host knows of how the tokens are spread: where most
// of them are idle a chunk of up to 127 tokens is taken one by one however far back it
// reads (100 tokens at position 30,000 in a table of one row 114 us, of 64 rows 616; 49
// at 8000 56 and 99).
constexpr int kPagedPlanTokens = 48;  // beyond one for each sequence
bool planned(int T, int n_seq) { return T >= kAttnTile || T - n_seq >= kPagedPlanTokens; }

// Workspace of moe_paged_attend.
struct PagedWs {
    size_t n_list, count, list, before, head, tiles, unit_count, part, unit_part, total;
};

PagedWs paged_ws(int64_t T) {
    auto up = [](size_t v) { return (v + 255) & ~size_t(255); };
    PagedWs L{};
    size_t o = 0;
    L.n_list = o; o += up(2 * 4);
    L.count = o; o += up(2 * kPagedMaxCtas * 4);
    L.list = o; o += up((size_t)T * 4);
    L.before = o; o += up(((size_t)T + 1) * 8);
    L.head = o; o += up(sizeof(AttnPlanHead));
    L.tiles = o; o += up((size_t)(T / kPagedTileMinRows) * sizeof(int4));
    L.unit_count = o; o += up(2 * kPagedUnitParts * 4);
    L.part = o; o += up(kPagedPartFloats * 4);
    // (a call of fewer tokens is not sorted, whatever its table)
    L.unit_part = o; o += planned((int)T, 1) ? up(kPagedUnitPartFloats * 4) : 0;
    L.total = o;
    return L;
}

template <typename P>
P *at(void *ws, size_t off) {
    return reinterpret_cast<P *>(static_cast<char *>(ws) + off);
}

cudaError_t attend(const PagedAttn &a, void *ws, cudaStream_t st) {
    const PagedWs L = paged_ws(a.T);
    PagedList l{at<int>(ws, L.n_list), at<int>(ws, L.n_list) + 1, at<int>(ws, L.list),
                at<long long>(ws, L.before), at<int>(ws, L.count)};
    PlanArgs pa{a.seq, a.pos, a.pv.n_seq, a.pv.max_pages << a.pv.shift, {}};
    static_assert(kAttnTile <= kPagedSmall, "a call that is not sorted needs no list");
    const bool sorted = planned(a.T, a.pv.n_seq);
    if (sorted)
        pa.plan = AttnPlan{at<AttnPlanHead>(ws, L.head), at<int4>(ws, L.tiles), l.list};
    {
        int T = a.T;
        PageView pv = a.pv;
        const int32_t *seq = a.seq, *pos = a.pos;
        int *unit_count = at<int>(ws, L.unit_count);
        void *args[] = {&T, &pv, &seq, &pos, &l, &pa, &unit_count};
        LaunchScope ls("paged_plan", st);
        cudaError_t e =
            launch_pdl((const void *)k_paged_plan, dim3(1), dim3(kPlanThreads), 0, st, args);
        if (e != cudaSuccess) return e;
    }
    if (sorted) {
        cudaError_t e = launch_paged_prefill_tc(a, pa.plan, at<float>(ws, L.unit_part),
                                                at<int>(ws, L.unit_count), st);
        if (e != cudaSuccess) return e;
    }
    return launch_paged_decode_tc(a, l, at<float>(ws, L.part), !sorted, st);
}

}  // namespace

moe_status check_paged(const moe_sa_dims *d, const moe_paged_dims *pd) {
    size_t n = 0;
    moe_status s = moe_sa_workspace_size(d, 0, &n);  // the shape's own limits
    if (s != MOE_OK) return s;
    if (!pd) return MOE_ERR_INVALID_ARG;
    if (pd->n_pages < 1 || pd->n_seq < 1 || pd->max_pages < 1 || pd->page_size < 1)
        return MOE_ERR_INVALID_ARG;
    if (pd->page_size != 16 && pd->page_size != 32 && pd->page_size != 64 && pd->page_size != 128)
        return MOE_ERR_UNSUPPORTED;
    // (a cache row's number is a TMA coordinate; the tiles of kPagedSmall tokens are
    // counted in 32 bits)
    if ((int64_t)pd->n_pages * d->n_kv_heads * pd->page_size > (1LL << 31) - 1 ||
        (int64_t)pd->max_pages * pd->page_size > 1LL << 30)
        return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

moe_status check_paged_call(const moe_sa_dims *d, const moe_paged_dims *pd, int32_t T,
                            const int32_t *seq, const int32_t *pos, const int32_t *table,
                            const void *kp, const void *vp, const float *ks, const float *vs) {
    moe_status s = check_paged(d, pd);
    if (s != MOE_OK) return s;
    if (T < 0 || T > kMaxSaTokens) return MOE_ERR_INVALID_ARG;
    if (T > 0 && (!ok_ptr(seq) || !ok_ptr(pos) || !ok_ptr(table) || !ok_ptr(kp) || !ok_ptr(vp) ||
                  !ok_ptr(ks) || !ok_ptr(vs)))
        return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

cudaError_t launch_paged_append(const moe_sa_dims &d, const moe_paged_dims &pd, int T,
                                const float *qkv, int n_part, long long part_stride,
                                const ProjSplit &split, const int32_t *seq, const int32_t *pos,
                                const int32_t *table, void *q, void *kp, void *vp, float *ks,
                                float *vs, cudaStream_t st) {
    const QkvRows rows{qkv, (d.n_heads + 2 * d.n_kv_heads) * kPagedDh, T, n_part, part_stride, split};
    return launch_append(rows, n_part == 1 ? kInF32 : kInParts, d, pd, seq, pos, table, q, kp, vp,
                         ks, vs, st);
}

cudaError_t launch_paged_attend(const moe_sa_dims &d, const moe_paged_dims &pd, int T,
                                const void *q, const int32_t *seq, const int32_t *pos,
                                const int32_t *table, const void *kp, const void *vp,
                                const float *ks, const float *vs, void *ctx, void *ws,
                                cudaStream_t st) {
    const PagedAttn a{T,
                      d.n_heads,
                      d.n_kv_heads,
                      pd.page_size,
                      PageView{table, pd.n_seq, pd.max_pages, pd.n_pages,
                               31 - __builtin_clz(pd.page_size)},
                      seq,
                      pos,
                      q,
                      kp,
                      vp,
                      ks,
                      vs,
                      ctx};
    return attend(a, ws, st);
}

}  // namespace moe

using namespace moe;

extern "C" {

moe_status moe_paged_workspace_size(const moe_sa_dims *dims, int32_t max_tokens, size_t *bytes) {
    size_t n = 0;
    moe_status s = moe_sa_workspace_size(dims, 0, &n);
    if (s != MOE_OK) return s;
    if (!bytes || max_tokens < 0 || max_tokens > kMaxSaTokens) return MOE_ERR_INVALID_ARG;
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
    return cuda_status(launch_paged_attend(*dims, *paged, T, q, seq, pos, page_table, k_pages,
                                           v_pages, k_scale, v_scale, ctx, ws,
                                           (cudaStream_t)stream));
}

}  // extern "C"
