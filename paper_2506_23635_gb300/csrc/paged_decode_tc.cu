// Attention of single tokens over the paged 8-bit cache on the tcgen05 tensor
// cores.
//
// The cache's e4m3 tiles are the matrix instructions' operands as they lie in
// memory; what is multiplied with them, queries and probabilities, is split
// into e4m3 terms that carry its precision, each a column of its own:
//
//   S^T = K Q^T       M = 128 positions, N = 16: columns h the first terms of
//                     the group's (up to 8) query heads, 8 + h the second, 16
//                     times as large; K = 128 dims.  A bf16 query scaled by a power
//                     of two so that its row's largest is in [128, 256) is the sum
//                     of its two terms but for 2^-21 of that largest.
//   O^T += V^T P^T    M = 128 dims, N = 32: columns 8 i + h the i-th term of head
//                     h's probabilities, 16^i times as large; K = 128 positions; V
//                     as it lies in the page (dims contiguous: an MN-major
//                     operand).  Four terms of four bits: 2^-16 of a probability,
//                     2^-30 of the largest.
//
// Decoding the tiles to 16 bits instead would write and read two more bytes of
// shared memory for each of theirs, 118 of the 128 bytes a clock that an SM
// moves there at the rate HBM delivers.
//
// The scale of a position's key page multiplies its score, that of its value
// page its probability (before the split: p vs against the largest p vs so
// far), so scales may be any positive numbers.  The row sum takes p itself.
//
// The position tiles of every listed (token, key/value head), token by token,
// are one list, of which each CTA (two an SM) takes an equal contiguous share,
// so every SM streams the same number of bytes whatever the sequences' lengths.
// A share is a run of pieces: the end of one (token, head)'s tiles, whole ones,
// the start of another's.  A (token, head) in one share is written to ctx at
// once; otherwise every share with a piece of it leaves (base, sum) and O^T in the
// workspace and, its share done, counts itself on the (token, head)'s counter; the
// one that counts last merges the pieces in order (no CTA waits for another,
// and the result depends on no order).
//
//   warp 0      a tile's pages from the table, their key and value rows by TMA
//               (a box a page, its lanes side by side) into three-stage rings,
//               their scales and the tile's description into a ring;
//   warp 1      tensor memory and the MMAs: S_{j+1} is issued before P_j V_j;
//   warps 2-5   softmax, one thread per position: a per-head base-2 exponent base
//               that moves only when a value passes it by more than 1.75 (then
//               O^T is rescaled in tensor memory, a thread its dim's row); the
//               four terms of its probabilities, 32 bytes, go to P_j, positions
//               as rows (MN-major, 32-byte swizzle); rows of V_j that hold no
//               position of the token, or whose scale is zero, are zeroed (0 x NaN is
//               NaN);
//   warp 6      the next piece's queries, split into terms.
//
// Every wait is bounded (ptx.cuh); once one gives up the thread skips the later
// waits and the kernel ends.
#include <math.h>

#include <algorithm>

#include "paged.cuh"

namespace moe {
namespace {

using namespace tc;

constexpr int kPdThreads = 7 * 32;
constexpr int kPdStages = 3;
constexpr int kPdRing = 8;  // tile descriptions
constexpr int kPdSmall = kPagedSmall;
// parts that one CTA merges: more are merged in groups first
constexpr int kPdGroup = 18;
static_assert(kPagedMaxCtas <= kPdGroup * kPdGroup && kPdGroup <= 32, "two levels of merging");
constexpr int kPdMaxG = kPagedMaxGroup;
constexpr int kPdMaxPages = kPagedTile / 16;  // pages of a tile at most
constexpr uint32_t kPdTile = kPagedTile * kPagedDh;  // 16 KB
constexpr uint32_t kPdQ = 16 * kPagedDh;             // 2 KB
constexpr uint32_t kPdP = kPagedTile * 32;           // 4 KB
constexpr uint32_t kPdOffK = 0;
constexpr uint32_t kPdOffV = kPdOffK + kPdStages * kPdTile;
constexpr uint32_t kPdOffQ = kPdOffV + kPdStages * kPdTile;
constexpr uint32_t kPdOffP = kPdOffQ + 2 * kPdQ;
constexpr uint32_t kPdOffHdr = kPdOffP + 2 * kPdP;
constexpr uint32_t kPdHdrBytes = 4096;
constexpr size_t kPdSmem = 1024 + kPdOffHdr + kPdHdrBytes;
static_assert(2 * (kPdSmem + 1024) <= 228 * 1024, "two CTAs an SM");
// kind::f8f6f4: e4m3 A and B, fp32 D, M = 128
constexpr uint32_t kPdIdesc = (1u << 4) | ((uint32_t)(kPagedTile >> 4) << 24);
constexpr uint32_t kPdIdescQK = kPdIdesc | ((16u >> 3) << 17);  // both K-major, N = 16
// both MN-major (bits 15, 16), N = 32
constexpr uint32_t kPdIdescPV = kPdIdesc | ((32u >> 3) << 17) | (1u << 15) | (1u << 16);
constexpr uint32_t kPdTmemCols = 64;
constexpr uint32_t kPdColS = 0, kPdColO = 32;  // S^T twice 16 columns, O^T 32
// probabilities are 2^(kPdTop) at the exponent base: with values up to 1.75 past
// it at most 2^8.75, inside e4m3's 448, and as far above its smallest as can be
constexpr float kPdTop = 7.f, kPdSlack = 1.75f;
constexpr float kPdNone = -1e30f;  // base of nothing

enum : int { kPdFirst = 1, kPdLast = 2, kPdWhole = 4, kPdEnd = 8, kPdClear = 16 };

struct PdDesc {
    int tile;     // -1: the share has ended
    int tg;       // token * Hkv + key/value head
    int n;        // positions the token attends to
    int flags;    // kPdFirst, kPdLast: of its piece; kPdWhole: the piece is the whole
                  // (token, head); kPdEnd: of its share; kPdClear: some value rows count as
                  // zeros (no position there, or a scale of zero)
    int b0, parts;  // not whole: the first share with a piece of it, and how many have one
    unsigned valid;  // bit i: page i of the tile holds positions
    int pad;
    float ks[kPdMaxPages], vs[kPdMaxPages], lv[kPdMaxPages];  // scales, log2 of vs
};

struct PdHeader {
    uint64_t k_full[kPdStages], k_empty[kPdStages];
    uint64_t v_full[kPdStages], v_empty[kPdStages];
    uint64_t s_full[2], s_empty[2];   // S_j written; read by the softmax warps
    uint64_t p_ready[2], p_empty[2];  // P_j written; P_j V_j finished
    uint64_t q_full[2], q_empty[2];   // a piece's queries written; read, and its scales
    uint64_t t_full[kPdRing];         // description of tile j published
    uint64_t done;
    uint32_t tmem_base;
    int last;  // this CTA counted last
    float qs[2][kPdMaxG];  // queries: what a score is to be multiplied with
    float red[4][kPdMaxG];
    float lsum[4][kPdMaxG];
    alignas(16) PdDesc desc[kPdRing];
    // a call of up to kPdSmall tokens, all of them listed: their sequences,
    // positions attended to, and the tiles of those ahead of each
    int seq[kPdSmall], n[kPdSmall], before[kPdSmall + 1];
};
static_assert(sizeof(PdHeader) <= kPdHdrBytes, "header");

__device__ __forceinline__ float pd_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Shared-memory descriptors.  Their upper half: 128-byte swizzle, 8 rows 1024 bytes
// apart (queries and keys, K-major; values, MN-major: the next 8 rows, of k), and
// 32-byte swizzle, 8 rows 256 bytes apart (probabilities, MN-major); the lower one's
// field beside the address.  No operand is wider than a row.
constexpr uint32_t kPdDescHi = (1024 >> 4) | 1u << 14 | 2u << 29;
constexpr uint32_t kPdDescPHi = (256 >> 4) | 1u << 14 | 6u << 29;
constexpr uint32_t kPdDescLo = 1u << 16;

// One lane of the warp, always the same.
__device__ __forceinline__ bool pd_elect() {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r));
    return r != 0;
}

// D[tmem] (+)= A[smem] * B[smem], 8-bit operands, one instruction of K = 32; a, b:
// the descriptors' lower halves.
__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint32_t a, uint32_t b, uint32_t b_hi,
                                       uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "mov.b64 da, {%1, %4};\n\tmov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a), "r"(b), "r"(idesc), "r"(kPdDescHi), "r"(b_hi), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ int pd_acquire(const int *p) {
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// What has been acquired, for the TMA loads that follow.
__device__ __forceinline__ void pd_fence_proxy_async() {
    asm volatile("fence.proxy.async.global;" ::: "memory");
}

// A whole warp's wait: the answer is the same in every lane.
__device__ __forceinline__ bool pd_wait(uint64_t *bar, uint32_t parity, unsigned *err) {
    return __all_sync(0xffffffffu, ptx::mbar_wait(bar, parity, err));
}

template <int N>
__device__ __forceinline__ void pd_tmem_ld(uint32_t taddr, float (&v)[N]);
template <>
__device__ __forceinline__ void pd_tmem_ld<32>(uint32_t taddr, float (&v)[32]) {
    tmem_ld32(taddr, v);
}
template <>
__device__ __forceinline__ void pd_tmem_ld<16>(uint32_t taddr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ void pd_tmem_st32(uint32_t taddr, const float (&v)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]),
        "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]),
        "f"(v[15]), "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]),
        "f"(v[22]), "f"(v[23]), "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]),
        "f"(v[29]), "f"(v[30]), "f"(v[31])
        : "memory");
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ float pd_warp_max(float v) {
    float m;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
    return m;
}

// Barrier over the softmax threads that also tells whether any of them had p.
__device__ __forceinline__ bool pd_any(bool p) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)p)
        : "memory");
    return r != 0;
}

// Shares of W tiles among G CTAs: CTA c starts at tile W c / G, and tile x is
// in CTA ((x + 1) G - 1) / W.
__device__ __forceinline__ long long pd_start(long long W, int c, int G) {
    if (W < (1 << 22)) return (unsigned)W * (unsigned)c / (unsigned)G;
    return W * c / G;
}
__device__ __forceinline__ int pd_owner(long long x, long long W, int G) {
    if (W < (1 << 22)) return (int)((((unsigned)x + 1u) * (unsigned)G - 1u) / (unsigned)W);
    return (int)(((x + 1) * G - 1) / W);
}
static_assert(kPagedMaxCtas < 1024, "the 32-bit products of pd_start and pd_owner");

// The listed tokens: those of the plan, or all of a small call (in shared
// memory, so that nothing waits for another kernel).
struct PdTokens {
    const PagedList &l;
    const PdHeader *hd;
    const int32_t *seq, *pos;
    const PageView &pv;
    int T;  // of a small call; 0: as listed

    __device__ __forceinline__ int count() const { return T > 0 ? T : __ldcg(l.n_list); }
    __device__ __forceinline__ long long before(int i) const {
        return T > 0 ? hd->before[i] : __ldcg(&l.before[i]);
    }
    __device__ __forceinline__ int token(int i) const { return T > 0 ? i : __ldcg(&l.list[i]); }
};

// Where a share begins, and the walk through its (token, head)s.
struct PdWalk {
    long long W;
    int n_list, n_share, Hkv;
    long long lo, hi;     // the share's tiles
    long long first;      // list's tile at which the present (token, head) begins
    int i, g, nt;         // present list entry, key/value head, its tiles
};

// The last entry with before(i) * Hkv <= x, by a warp.
__device__ __forceinline__ int pd_find(const PdTokens &l, int n, int Hkv, long long x) {
    const int lane = threadIdx.x & 31;
    int lo = 0, len = n;  // the answer is in [lo, lo + len)
    while (len > 1) {
        const int step = (len + 31) / 32;
        const int i = lo + lane * step;
        const bool le = lane * step < len && l.before(i) * Hkv <= x;
        const uint32_t m = __ballot_sync(0xffffffffu, le);
        const int k = 31 - __clz(m);  // (entry lo itself always is)
        lo += k * step;
        len = min(step, len - k * step);
    }
    return lo;
}

__device__ __forceinline__ PdWalk pd_begin(const PdTokens &l, int Hkv, int cta, int G) {
    PdWalk w;
    w.Hkv = Hkv;
    w.n_list = l.count();
    w.W = w.n_list > 0 ? l.before(w.n_list) * Hkv : 0;
    w.n_share = (int)min((long long)G, w.W);
    w.lo = w.hi = 0;
    if (cta >= w.n_share) return w;
    w.lo = pd_start(w.W, cta, w.n_share);
    w.hi = pd_start(w.W, cta + 1, w.n_share);
    w.i = pd_find(l, w.n_list, Hkv, w.lo);
    const long long b = l.before(w.i);
    w.nt = (int)(l.before(w.i + 1) - b);
    const long long in = w.lo - b * Hkv;
    w.g = in < (1 << 30) ? (int)((unsigned)in / (unsigned)w.nt) : (int)(in / w.nt);
    w.first = b * Hkv + (long long)w.g * w.nt;
    return w;
}

// On to the next (token, head).
__device__ __forceinline__ void pd_next(const PdTokens &l, PdWalk &w) {
    w.first += w.nt;
    if (++w.g == w.Hkv) {
        w.g = 0;
        if (w.first < w.hi) do {
                ++w.i;
                w.nt = (int)(l.before(w.i + 1) - l.before(w.i));
            } while (w.nt == 0);
    }
}

__device__ __forceinline__ float pd_mean(float a, float s) { return s == 0.f ? 0.f : a / s; }

// Up to 32 parts in the workspace merged in order: part k lies in slot slot(k).
// A warp of the four takes every fourth head, a lane four dims; eight parts' loads
// go out together, past L1.  The result goes to dst (the group's heads in ctx), or
// to the slot `into`, which may be one of them (only the warp itself reads its
// heads there).  (A thread a dim with all heads, three parts at a time: 3.4 us for
// 8 parts of 6 heads, and one token over 2048 positions 11.7 us instead of 10.4.)
template <int G, typename Slot>
__device__ __forceinline__ void pd_merge(const float *part, Slot slot, int parts, int w, bf16 *dst,
                                         float *into) {
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int h = w; h < G; h += 4) {
        float2 bl = make_float2(kPdNone, 0.f);
        if (lane < parts)
            bl = __ldcg(reinterpret_cast<const float2 *>(part + (size_t)slot(lane) * kPagedSlot +
                                                         kPdMaxG * 128 + 2 * h));
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        float M = 0.f, wt = 0.f, S = 0.f;
#pragma unroll 1
        for (int q0 = 0; q0 < parts; q0 += 8) {
            float4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int q = min(q0 + u, parts - 1);
                v[u] = __ldcg(reinterpret_cast<const float4 *>(
                    part + (size_t)slot(q) * kPagedSlot + h * 128 + 4 * lane));
            }
            if (q0 == 0) {
                M = pd_warp_max(bl.x);
                wt = lane < parts ? pd_exp2(bl.x - M) : 0.f;
                S = warp_sum(wt * bl.y);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float c = __shfl_sync(0xffffffffu, wt, (q0 + u) & 31);
                if (q0 + u >= parts) continue;
                acc.x = fmaf(c, v[u].x, acc.x);
                acc.y = fmaf(c, v[u].y, acc.y);
                acc.z = fmaf(c, v[u].z, acc.z);
                acc.w = fmaf(c, v[u].w, acc.w);
            }
        }
        if (into) {
            __syncwarp();
            *reinterpret_cast<float4 *>(into + h * 128 + 4 * lane) = acc;
            if (lane == 0)
                *reinterpret_cast<float2 *>(into + kPdMaxG * 128 + 2 * h) = make_float2(M, S);
            continue;
        }
        const __nv_bfloat162 lo = __floats2bfloat162_rn(pd_mean(acc.x, S), pd_mean(acc.y, S));
        const __nv_bfloat162 hi = __floats2bfloat162_rn(pd_mean(acc.z, S), pd_mean(acc.w, S));
        *reinterpret_cast<uint2 *>(dst + h * kPagedDh + 4 * lane) =
            make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
    }
}

struct PdArgs {
    int T;  // tokens of a small call, all of them listed; 0: as the plan lists them
    int Hq, Hkv;
    PageView pv;
    PagedList list;
    const int32_t *seq, *pos;
    const bf16 *q;
    const float *ks, *vs;
    bf16 *ctx;
    float *part;
    unsigned *err;
};

template <int G>
__global__ void __launch_bounds__(kPdThreads, 2)
k_paged_decode_tc(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  const PdArgs a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    PdHeader *hd = reinterpret_cast<PdHeader *>(smem + kPdOffHdr);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cta = (int)blockIdx.x, n_cta = (int)gridDim.x, Hkv = a.Hkv;
    unsigned *err = a.err;
    ptx::launch_dependents();
    const bool small = a.T > 0;
    // Beside the prefill attention: that one starts when the plan is complete and lets
    // this one start then, so what the plan has released, its own list and all that
    // was complete ahead of it, is acquired from it, not waited for (a wait for
    // the prefill: 512 tokens at position 5000 beside 24 others 94 us, 117 so).
    if (!small) {
        int n = pd_acquire(a.list.released) - 1;
        if (n < 0) {
            ptx::grid_dependency_wait();
            n = __ldcg(a.list.n_list);
        }
        pd_fence_proxy_async();
        // (nothing listed beside the tiles: 2000 tokens of 16 heads 40.9 us, 40.3 so)
        if (n == 0) {
            if (cta == n_cta - 1) ptx::grid_dependency_wait();
            return;
        }
    }
    if (threadIdx.x == 0) {
        for (int b = 0; b < kPdStages; ++b) {
            ptx::mbar_init(&hd->k_full[b], 1);
            ptx::mbar_init(&hd->k_empty[b], 1);
            ptx::mbar_init(&hd->v_full[b], 1);
            ptx::mbar_init(&hd->v_empty[b], 1);
        }
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(&hd->s_full[b], 1);
            ptx::mbar_init(&hd->s_empty[b], 4);
            ptx::mbar_init(&hd->p_ready[b], 4);
            ptx::mbar_init(&hd->p_empty[b], 1);
            ptx::mbar_init(&hd->q_full[b], 1);
            ptx::mbar_init(&hd->q_empty[b], 5);
        }
        for (int b = 0; b < kPdRing; ++b) ptx::mbar_init(&hd->t_full[b], 1);
        ptx::mbar_init(&hd->done, 1);
        ptx::fence_barrier_init();
        ptx::prefetch_tmap(&tmK);
        ptx::prefetch_tmap(&tmV);
    }
    if (warp == 1) tmem_alloc(&hd->tmem_base, kPdTmemCols);
    if (small) ptx::grid_dependency_wait();
    if (warp == 2 && small) {
        // the tiles before each token; one outside the table has none
        constexpr int E = kPdSmall / 32;
        int nt[E], sum = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int t = E * lane + e;
            const int sq = t < a.T ? a.seq[t] : -1, p = t < a.T ? a.pos[t] : -1;
            const bool in = a.pv.inside(sq, p);
            hd->seq[t] = sq;
            hd->n[t] = in ? p + 1 : 0;
            nt[e] = in ? p / kPagedTile + 1 : 0;
            sum += nt[e];
        }
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        int run = incl - sum;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            hd->before[E * lane + e] = run;
            run += nt[e];
        }
        if (lane == 31) hd->before[kPdSmall] = run;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const PdTokens tokens{a.list, hd, a.seq, a.pos, a.pv, a.T};
    const uint32_t tmem = hd->tmem_base;
    const uint32_t sbase = ptx::smem_u32(smem);

    if (warp == 0) {
        // ------------------------------------------------------------ pages
        const uint64_t pol = ptx::policy_evict_first();  // a tile is read once
        PdWalk w = pd_begin(tokens, Hkv, cta, n_cta);
        const int shift = a.pv.shift, per = kPagedTile >> shift;  // pages of a tile
        const uint32_t page_bytes = (uint32_t)kPagedDh << shift;
        bool good = true;
        int j = 0, sent_k = 0, sent_v = 0, of = -1;
        // a tile of the walk, looked up one ahead of its turn
        struct Ahead {
            int tok, sq, n, g, tile, nt;
            long long first;
            int entry;  // its page `lane`, as the table has it
        } next = {};
        auto look = [&](long long x) {
            if (x == w.first + w.nt) pd_next(tokens, w);
            if (w.i != of) {
                of = w.i;
                next.tok = tokens.token(w.i);
                next.sq = small ? hd->seq[w.i] : a.seq[next.tok];
                const int p = small ? hd->n[w.i] - 1 : a.pos[next.tok];
                next.n = p + 1;  // (a token with tiles lies inside the table)
            }
            next.g = w.g;
            next.first = w.first;
            next.nt = w.nt;
            next.tile = (int)(x - w.first);
            const int p = next.tile * kPagedTile + (lane << shift);
            next.entry = lane < per && p < next.n
                             ? a.pv.table[(size_t)next.sq * a.pv.max_pages + (p >> shift)]
                             : -1;
        };
        if (w.lo < w.hi) look(w.lo);
        for (long long x = w.lo; x < w.hi; ++x, ++j) {
            const Ahead c = next;
            if (x + 1 < w.hi) look(x + 1);
            const int pg = c.entry >= 0 && c.entry < a.pv.n_pages ? c.entry : -1;
            const int left = c.n - c.tile * kPagedTile;  // positions from the tile's first on
            if (pg < 0 && lane < per && (lane << shift) < left) set_error(err, kErrIndex);
            float ks = 0.f, vs = 0.f;
            if (pg >= 0) {
                // (not __ldg: its loads are outside of what an acquire orders)
                ks = __ldcg(a.ks + (size_t)pg * Hkv + c.g);
                vs = __ldcg(a.vs + (size_t)pg * Hkv + c.g);
            }
            const unsigned valid = __ballot_sync(0xffffffffu, pg >= 0);
            const uint32_t bytes = (uint32_t)__popc(valid) * page_bytes;
            const int st = j % kPdStages;
            const uint32_t ph = (uint32_t)(j / kPdStages) & 1u;
            const int row = (pg * Hkv + c.g) << shift;
            if (!(good = pd_wait(&hd->k_empty[st], ph ^ 1u, err))) break;
            if (lane == 0) ptx::mbar_arrive_expect_tx(&hd->k_full[st], bytes);
            __syncwarp();
            sent_k = j + 1;
            if (pg >= 0)
                ptx::tma_load_2d(smem + kPdOffK + st * kPdTile + lane * page_bytes, &tmK, 0, row,
                                 &hd->k_full[st], pol);
            if (!(good = pd_wait(&hd->v_empty[st], ph ^ 1u, err))) break;
            if (lane == 0) ptx::mbar_arrive_expect_tx(&hd->v_full[st], bytes);
            __syncwarp();
            sent_v = j + 1;
            if (pg >= 0)
                ptx::tma_load_2d(smem + kPdOffV + st * kPdTile + lane * page_bytes, &tmV, 0, row,
                                 &hd->v_full[st], pol);
            PdDesc *d = &hd->desc[j % kPdRing];
            // (asked for after the loads: the scales are long in coming)
            const unsigned sound = __ballot_sync(0xffffffffu, pg >= 0 && vs != 0.f);
            if (lane < per) {
                d->ks[lane] = ks;
                d->vs[lane] = vs;
                // (the exponent base takes scales below 2^-100, which
                // moe_paged_append does not give, and zero for 2^-100)
                d->lv[lane] = log2f(fmaxf(vs, 7.888609052210118e-31f));
            }
            if (lane == 0) {
                const bool whole = c.first >= w.lo && c.first + c.nt <= w.hi;
                const bool first = c.tile == 0 || x == w.lo;
                const bool last = c.tile == c.nt - 1 || x == w.hi - 1;
                d->tile = c.tile;
                d->tg = c.tok * Hkv + c.g;
                d->n = c.n;
                d->valid = valid;
                d->flags = (first ? kPdFirst : 0) | (last ? kPdLast : 0) | (whole ? kPdWhole : 0) |
                           (x == w.hi - 1 ? kPdEnd : 0) |
                           (left < kPagedTile || (int)__popc(sound) < per ? kPdClear : 0);
                if (!whole && last) {
                    d->b0 = pd_owner(c.first, w.W, w.n_share);
                    d->parts = pd_owner(c.first + c.nt - 1, w.W, w.n_share) - d->b0 + 1;
                }
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&hd->t_full[j % kPdRing]);
        }
        // the end of the share, also where a wait gave up
        if (lane == 0) {
            hd->desc[j % kPdRing].tile = -1;
            ptx::mbar_arrive(&hd->t_full[j % kPdRing]);
            // loads in flight land before the block can exit
            for (int u = max(0, sent_k - kPdStages); u < sent_k; ++u)
                ptx::mbar_wait(&hd->k_full[u % kPdStages], (uint32_t)(u / kPdStages) & 1u, err);
            for (int u = max(0, sent_v - kPdStages); u < sent_v; ++u)
                ptx::mbar_wait(&hd->v_full[u % kPdStages], (uint32_t)(u / kPdStages) & 1u, err);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA
        // The whole warp runs it and one lane issues: operands that are the same in
        // every lane by the code go to uniform registers, which the instructions take
        // them from, at once (a branch of one lane's moves each there first).
        bool good = true;
        int piece = -1;
        uint32_t acc = 0, acc1 = 0;  // tile j, tile j - 1 adds to O
        const bool lead = pd_elect();
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        const uint32_t k0 = ((sbase + kPdOffK) >> 4) | kPdDescLo, q0 = ((sbase + kPdOffQ) >> 4) | kPdDescLo;
        const uint32_t v0 = ((sbase + kPdOffV) >> 4) | kPdDescLo, p0 = ((sbase + kPdOffP) >> 4) | kPdDescLo;
#pragma unroll 1
        for (int j = 0; good; ++j) {
            if (!(good = pd_wait(&hd->t_full[j % kPdRing], (uint32_t)(j / kPdRing) & 1u, err))) break;
            const PdDesc *d = &hd->desc[j % kPdRing];
            const bool more = __shfl_sync(0xffffffffu, d->tile, 0) >= 0;
            if (more) {
                const int flags = __shfl_sync(0xffffffffu, d->flags, 0), st = j % kPdStages;
                acc = flags & kPdFirst ? 0u : 1u;
                if (flags & kPdFirst) {
                    ++piece;
                    good = pd_wait(&hd->q_full[piece & 1], (uint32_t)(piece >> 1) & 1u, err);
                }
                good = good && pd_wait(&hd->k_full[st], (uint32_t)(j / kPdStages) & 1u, err) &&
                       pd_wait(&hd->s_empty[j & 1], ((uint32_t)(j >> 1) & 1u) ^ 1u, err);
                if (!good) break;
                tc_fence_after();
                if (lead) {
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_f8(tm + kPdColS + (j & 1) * 16, k0 + ((st * kPdTile) >> 4) + 2 * kk,
                               q0 + (((piece & 1) * kPdQ) >> 4) + 2 * kk, kPdDescHi, kPdIdescQK,
                               kk != 0);
                    mma_commit(&hd->s_full[j & 1]);
                    mma_commit(&hd->k_empty[st]);
                    if (flags & kPdLast) mma_commit(&hd->q_empty[piece & 1]);
                }
                __syncwarp();
            }
            if (j > 0) {  // P_{j-1} V_{j-1}
                const int u = j - 1, st = u % kPdStages;
                good = pd_wait(&hd->v_full[st], (uint32_t)(u / kPdStages) & 1u, err) &&
                       pd_wait(&hd->p_ready[u & 1], (uint32_t)(u >> 1) & 1u, err);
                if (!good) break;
                tc_fence_after();
                if (lead) {
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_f8(tm + kPdColO, v0 + ((st * kPdTile + kk * 32 * kPagedDh) >> 4),
                               p0 + (((u & 1) * kPdP + kk * 32 * 32) >> 4), kPdDescPHi, kPdIdescPV,
                               kk != 0 ? 1u : acc1);
                    mma_commit(&hd->p_empty[u & 1]);
                    mma_commit(&hd->v_empty[st]);
                }
                __syncwarp();
            }
            acc1 = acc;
            if (!more) break;
        }
        // every MMA has finished before tensor memory is freed
        if (lead) mma_commit(&hd->done);
        pd_wait(&hd->done, 0, err);
    } else if (warp == 6) {
        // ------------------------------------------------------------ queries
        PdWalk w = pd_begin(tokens, Hkv, cta, n_cta);
        bool good = true;
        for (int piece = 0; w.lo < w.hi && w.first < w.hi && good; ++piece) {
            const int tok = tokens.token(w.i);
            const bf16 *src = a.q + ((size_t)tok * a.Hq + w.g * G) * kPagedDh + 4 * lane;
            uint2 u[G];
#pragma unroll
            for (int h = 0; h < G; ++h) u[h] = *reinterpret_cast<const uint2 *>(src + h * kPagedDh);
            const int b = piece & 1;
            if (!(good = pd_wait(&hd->q_empty[b], ((uint32_t)(piece >> 1) & 1u) ^ 1u, err))) break;
            unsigned char *qb = smem + kPdOffQ + b * kPdQ;
#pragma unroll
            for (int h = 0; h < G; ++h) {
                float f[4];
                unpack_bf16x2(u[h].x, f[0], f[1]);
                unpack_bf16x2(u[h].y, f[2], f[3]);
                // (as integers: NaN is the largest)
                const uint32_t m2 = __vmaxu2(u[h].x & 0x7fff7fffu, u[h].y & 0x7fff7fffu);
                const uint32_t mb = __reduce_max_sync(0xffffffffu, max(m2 & 0xffffu, m2 >> 16)) << 16;
                // 2^(7 - x) for a largest of 2^x to 2^(x+1) (x >= -119: what
                // lies below does not count)
                const int e = min(max((int)(mb >> 23), 8), 254);
                const float up = __uint_as_float((uint32_t)(254 + 7 - e) << 23);
                float t1[4], t2[4];
                uint32_t w1 = 0, w2 = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    t1[i] = f[i] * up;
                    if (!(fabsf(f[i]) <= 3.402823466e38f)) t1[i] = __uint_as_float(0x7fffffffu);
                }
                w1 = e4m3x2(t1[0], t1[1]) | e4m3x2(t1[2], t1[3]) << 16;
                const float2 b0 = e4m3x2_to_float2(w1 & 0xffffu), b1 = e4m3x2_to_float2(w1 >> 16);
                t2[0] = (t1[0] - b0.x) * 16.f;
                t2[1] = (t1[1] - b0.y) * 16.f;
                t2[2] = (t1[2] - b1.x) * 16.f;
                t2[3] = (t1[3] - b1.y) * 16.f;
                w2 = e4m3x2(t2[0], t2[1]) | e4m3x2(t2[2], t2[3]) << 16;
                const uint32_t at = h * 128 + (((lane >> 2) ^ h) << 4) + (lane & 3) * 4;
                *reinterpret_cast<uint32_t *>(qb + at) = w1;
                *reinterpret_cast<uint32_t *>(qb + 1024 + at) = w2;
                // log2(e) / sqrt(128); NaN where the query is not finite, for keys under a
                // scale of zero
                if (lane == 0)
                    hd->qs[b][h] = mb < 0x7f800000u
                                       ? 0.12751743f * __uint_as_float((uint32_t)(e - 7) << 23)
                                       : __uint_as_float(0x7fffffffu);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&hd->q_full[b]);
            pd_next(tokens, w);
        }
        // tokens with no position (padding, or outside the table): zeros
        for (int i = cta; i < w.n_list; i += n_cta) {
            if (tokens.before(i + 1) != tokens.before(i)) continue;
            uint4 *row = reinterpret_cast<uint4 *>(a.ctx + (size_t)tokens.token(i) * a.Hq * kPagedDh);
            for (int c = lane; c < a.Hq * kPagedDh / 8; c += 32) row[c] = make_uint4(0u, 0u, 0u, 0u);
            const int t = tokens.token(i);
            if (lane == 0 && a.seq[t] >= 0) set_error(err, kErrIndex);
        }
    } else {
        // ------------------------------------------------------------ softmax
        const int qt = warp & 3;  // tensor-memory lane quarter
        const int r = qt * 32 + lane;
        const uint32_t lane_base = (uint32_t)(qt * 32) << 16;
        const uint32_t o_col = tmem + lane_base + kPdColO;
        float base[G], l[G], qs[G];
#pragma unroll
        for (int h = 0; h < G; ++h) {
            base[h] = kPdNone;
            l[h] = qs[h] = 0.f;
        }
        bool good = true;
        int piece = -1;
        // parts to count at the end of the share: of the (token, head) that it
        // begins inside, and of the one that it ends inside
        int pend_tg0 = 0, pend_b0 = 0, pend_parts0 = 0, pend_tg1 = 0, pend_b1 = 0, pend_parts1 = 0;
#pragma unroll 1
        for (int j = 0;; ++j) {
            // (a wait that gave up ends the loop of all four warps: they
            // meet in barriers)
            good = good && pd_wait(&hd->t_full[j % kPdRing], (uint32_t)(j / kPdRing) & 1u, err);
            const PdDesc *d = &hd->desc[j % kPdRing];
            const bool end = !good || d->tile < 0;
            const int flags = d->flags, n = d->n, pos0 = d->tile * kPagedTile;
            const int pi = r >> a.pv.shift;  // the position's page of the tile
            const float ks = d->ks[pi], vs = d->vs[pi], lv = d->lv[pi];
            const bool live = pos0 + r < n && ((d->valid >> pi) & 1u);
            const bool first = flags & kPdFirst;
            if (!end && first) {
                ++piece;
                good = pd_wait(&hd->q_full[piece & 1], (uint32_t)(piece >> 1) & 1u, err);
#pragma unroll
                for (int h = 0; h < G; ++h) {
                    qs[h] = hd->qs[piece & 1][h];
                    base[h] = kPdNone;
                    l[h] = 0.f;
                }
            }
            float s[G];
            bool past = first;
            if (!end) {
                good = good && pd_wait(&hd->s_full[j & 1], (uint32_t)(j >> 1) & 1u, err);
                __syncwarp();
                tc_fence_after();
                float v[16];
                pd_tmem_ld<16>(tmem + lane_base + kPdColS + (j & 1) * 16, v);
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&hd->s_empty[j & 1]);
#pragma unroll
                for (int h = 0; h < G; ++h) {
                    // (keys under a scale of zero are zeros, whatever they hold)
                    const float f = ks * qs[h];
                    s[h] = ks == 0.f ? f : fmaf(v[8 + h], 0.0625f, v[h]) * f;
                    past = past || (live && s[h] + lv > base[h] + kPdSlack);
                }
            }
            if (pd_any(past || end || !good)) {
                if (pd_any(end || !good)) break;  // all four warps together
#pragma unroll
                for (int h = 0; h < G; ++h) {
                    const float m = pd_warp_max(live ? s[h] + lv : kPdNone);
                    if (lane == 0) hd->red[qt][h] = m;
                }
                ptx::named_bar_sync(1, 128);
                float corr[G];
#pragma unroll
                for (int h = 0; h < G; ++h) {
                    const float m = fmaxf(fmaxf(hd->red[0][h], hd->red[1][h]),
                                          fmaxf(hd->red[2][h], hd->red[3][h]));
                    const float nb = fmaxf(base[h], m);
                    corr[h] = pd_exp2(base[h] - nb);
                    base[h] = nb;
                    l[h] *= corr[h];
                }
                if (!first) {
                    // P_{j-1} V_{j-1} has finished, P_j V_j waits for this warp
                    good = pd_wait(&hd->p_empty[(j - 1) & 1], (uint32_t)((j - 1) >> 1) & 1u, err);
                    __syncwarp();
                    tc_fence_after();
                    float o[32];
                    pd_tmem_ld<32>(o_col, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int h = 0; h < G; ++h) o[8 * i + h] *= corr[h];
                    pd_tmem_st32(o_col, o);
                }
            }
            // the probabilities' terms: byte 8 i + h
            uint32_t word[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) word[i] = 0u;
#pragma unroll
            for (int h = 0; h < G; h += 2) {
                float e0 = pd_exp2(s[h] - base[h] + kPdTop), e1 = 0.f;
                e0 = live ? e0 : 0.f;
                l[h] += e0;
                float w0 = live ? e0 * vs : 0.f, w1 = 0.f;
                if (h + 1 < G) {
                    e1 = pd_exp2(s[h + 1] - base[h + 1] + kPdTop);
                    e1 = live ? e1 : 0.f;
                    l[h + 1] += e1;
                    w1 = live ? e1 * vs : 0.f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t t = e4m3x2(w0, w1);
                    word[2 * i + (h >> 2)] |= t << (8 * (h & 3));
                    if (i < 3) {
                        const float2 b = e4m3x2_to_float2(t);
                        w0 = (w0 - b.x) * 16.f;
                        w1 = (w1 - b.y) * 16.f;
                    }
                }
            }
            // (P_{j-2} V_{j-2} has read the buffer)
            good = good && pd_wait(&hd->p_empty[j & 1], ((uint32_t)(j >> 1) & 1u) ^ 1u, err);
            {
                unsigned char *pb = smem + kPdOffP + (j & 1) * kPdP + r * 32;
                const uint32_t sw = (uint32_t)(r >> 2) & 1u;
                *reinterpret_cast<uint4 *>(pb + (sw << 4)) = make_uint4(word[0], word[1], word[2], word[3]);
                *reinterpret_cast<uint4 *>(pb + ((sw ^ 1u) << 4)) =
                    make_uint4(word[4], word[5], word[6], word[7]);
            }
            if (flags & kPdClear) {
                good = good &&
                       pd_wait(&hd->v_full[j % kPdStages], (uint32_t)(j / kPdStages) & 1u, err);
                unsigned char *vr = smem + kPdOffV + (j % kPdStages) * kPdTile + r * kPagedDh;
#pragma unroll
                for (int c = 0; c < kPagedDh; c += 16)
                    if (!live || vs == 0.f)
                        *reinterpret_cast<uint4 *>(vr + c) = make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async_smem();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&hd->p_ready[j & 1]);
            if (!(flags & kPdLast)) continue;

            // the end of a piece
            const int tg = d->tg;
            const bool whole = flags & kPdWhole;
            const int b0 = whole ? 0 : d->b0, parts = whole ? 0 : d->parts;
#pragma unroll
            for (int h = 0; h < G; ++h) {
                const float t = warp_sum(l[h]);
                if (lane == 0) hd->lsum[qt][h] = t;
            }
            good = good && pd_wait(&hd->p_empty[j & 1], (uint32_t)(j >> 1) & 1u, err);
            __syncwarp();
            tc_fence_after();
            float o[32];
            pd_tmem_ld<32>(o_col, o);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&hd->q_empty[piece & 1]);
            ptx::named_bar_sync(1, 128);
            float L[G];
#pragma unroll
            for (int h = 0; h < G; ++h) {
                L[h] = (hd->lsum[0][h] + hd->lsum[1][h]) + (hd->lsum[2][h] + hd->lsum[3][h]);
                o[h] = fmaf(fmaf(fmaf(o[24 + h], 0.0625f, o[16 + h]), 0.0625f, o[8 + h]), 0.0625f, o[h]);
            }
            const int t = tg / Hkv, g = tg - t * Hkv;
            bf16 *dst = a.ctx + ((size_t)t * a.Hq + g * G) * kPagedDh + r;
            if (whole) {
#pragma unroll
                for (int h = 0; h < G; ++h)
                    dst[h * kPagedDh] = __float2bfloat16_rn(pd_mean(o[h], L[h]));
            } else {
                // the piece that starts the (token, head) ends its CTA's share
                const int slot = cta == b0 ? 1 : 0;
                float *mine = a.part + (size_t)(2 * cta + slot) * kPagedSlot;
#pragma unroll
                for (int h = 0; h < G; ++h) {
                    mine[h * 128 + r] = o[h];
                    if (r == 0)
                        *reinterpret_cast<float2 *>(mine + kPdMaxG * 128 + 2 * h) =
                            make_float2(base[h], L[h]);
                }
                if (slot) pend_tg1 = tg, pend_b1 = b0, pend_parts1 = parts;
                else pend_tg0 = tg, pend_b0 = b0, pend_parts0 = parts;
            }
            if (!(flags & kPdEnd) || (pend_parts0 == 0 && pend_parts1 == 0)) continue;
            // the share is done: its parts are counted, and the CTA that counts
            // last on a (token, head) finds every part of it stored; more than
            // kPdGroup parts are counted and merged in groups of that many first
            // (200,001 positions of one head over 304 CTAs: 96 us, all parts by one
            // CTA, 22.7 so)
#pragma unroll 1
            for (int i = 0; i < 2; ++i) {
                const int parts2 = i ? pend_parts1 : pend_parts0;
                if (parts2 == 0) continue;
                const int b2 = i ? pend_b1 : pend_b0, tg2 = i ? pend_tg1 : pend_tg0;
                const int t2 = tg2 / Hkv, g2 = tg2 - t2 * Hkv;
                bf16 *dst2 = a.ctx + ((size_t)t2 * a.Hq + g2 * G) * kPagedDh;
                // part k: the first slot of CTA b2 + k, but its second where the
                // (token, head) starts
                auto slot = [&](int k) { return 2 * (b2 + k) + (k == 0 ? 1 : 0); };
                // the last of n to count on counter `at`, with all they stored
                auto last_of = [&](int at, int n) {
                    ptx::named_bar_sync(1, 128);
                    if (r == 0) {  // (releases what the barrier has ordered before it)
                        int old;
                        asm volatile("atom.add.acq_rel.gpu.s32 %0, [%1], 1;"
                                     : "=r"(old)
                                     : "l"(a.list.count + at)
                                     : "memory");
                        hd->last = old == n - 1;
                    }
                    ptx::named_bar_sync(1, 128);
                    return hd->last != 0;
                };
                if (parts2 > kPdGroup) {
                    const int k0 = (cta - b2) / kPdGroup * kPdGroup;
                    const int n = min(kPdGroup, parts2 - k0);
                    // (a counter by the group's last CTA: only the last one
                    // of a (token, head) may start another)
                    if (!last_of(kPagedMaxCtas + b2 + k0 + n - 1, n)) continue;
                    float *into = a.part + (size_t)slot(k0) * kPagedSlot;
                    pd_merge<G>(a.part, [&](int k) { return slot(k0 + k); }, n, warp - 2, nullptr, into);
                }
                const int groups = parts2 > kPdGroup ? (parts2 + kPdGroup - 1) / kPdGroup : parts2;
                if (!last_of(b2, groups)) continue;
                pd_merge<G>(
                    a.part, [&](int k) { return slot(parts2 > kPdGroup ? k * kPdGroup : k); },
                    groups, warp - 2, dst2, nullptr);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, kPdTmemCols);
    // this grid is complete only after what is ahead: one CTA sees to it (the others
    // would keep their SMs from those that wait for one: 512 tokens at position
    // 5000 beside 24 of up to 2048 positions 144 us, 126 so)
    if (!small && cta == n_cta - 1) ptx::grid_dependency_wait();
}

const void *pd_kernel(int G) {
    switch (G) {
        case 1: return (const void *)k_paged_decode_tc<1>;
        case 2: return (const void *)k_paged_decode_tc<2>;
        case 3: return (const void *)k_paged_decode_tc<3>;
        case 4: return (const void *)k_paged_decode_tc<4>;
        case 5: return (const void *)k_paged_decode_tc<5>;
        case 6: return (const void *)k_paged_decode_tc<6>;
        case 7: return (const void *)k_paged_decode_tc<7>;
        default: return (const void *)k_paged_decode_tc<8>;
    }
}

}  // namespace

cudaError_t launch_paged_decode_tc(const PagedAttn &a, const PagedList &l, float *part, bool small,
                                   cudaStream_t st) {
    const int G = a.Hq / a.Hkv;
    CUtensorMap mk, mv;
    if (!paged_map(&mk, a.kp, a, true) || !paged_map(&mv, a.vp, a, true))
        return cudaErrorInvalidValue;
    const void *kern = pd_kernel(G);
    static SmemOnce once[kPdMaxG];
    cudaError_t e = once[G - 1].set(kern, kPdSmem);
    if (e != cudaSuccess) return e;
    PdArgs pa{small ? a.T : 0, a.Hq, a.Hkv, a.pv, l, a.seq, a.pos,
              static_cast<const bf16 *>(a.q), a.ks, a.vs, static_cast<bf16 *>(a.ctx), part,
              device_info().err};
    void *args[] = {&mk, &mv, &pa};
    // as many CTAs as the largest positions give tiles
    const long long most = (long long)a.T * a.Hkv *
                           (((long long)a.pv.max_pages * a.page_size + kPagedTile - 1) / kPagedTile);
    const int ctas = std::min(2 * device_info().sm_count, kPagedMaxCtas);
    LaunchScope ls("paged_decode_tc", st);
    return launch_pdl(kern, dim3((unsigned)std::min<long long>(most, ctas)), dim3(kPdThreads), kPdSmem,
                      st, args);
}

}  // namespace moe
