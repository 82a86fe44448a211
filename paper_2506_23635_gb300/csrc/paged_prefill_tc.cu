// Causal attention of prefill tiles over the paged 8-bit cache on the tcgen05
// tensor cores.
//
// Tiles and units are those of attn_tc.cu: a tile is 16 to 128 consecutive
// positions p0 .. p0 + rows - 1 of one sequence, a unit a (tile, pair of query
// heads of one key/value head) over cache positions 0 .. p0 + rows - 1, taken by
// one CTA an SM from a counter, longest first; the two heads share every key and
// value tile of 128 positions and take turns on the tensor cores.  Where that leaves
// SMs idle a unit is one head's, or a part of the positions, merged by the part
// that ends last.
//
// 128 queries share a tile, so its e4m3 numbers are decoded once, to fp16, which
// holds them exactly (half an instruction and four bytes of shared-memory traffic
// each, against 2 x 256 multiply-adds); queries scaled by a power of two (the largest
// of a row in [2^14, 2^15)) are exact in fp16 too, and so is what the products S =
// Q K^T are made of.  A score is multiplied with its key page's scale, a
// probability with its value page's (log2 of it in the exponent) before it is rounded
// to fp16: 2^-11 of it, one term, where bf16 would need two.  The row sum takes the
// probability itself.
//
//   warp 0      tensor memory (two score tiles S, a head each or one head's by
//               turns, and an output tile O per head, of 128 columns) and the MMAs:
//               S_j = Q K_j^T, and once P_j has taken S_j's place, O += P_j V_j with
//               P_j read from tensor memory and V_j MN-major as it lies;
//   warp 1      a tile's pages by TMA, as they are, its scales;
//   warps 2-4   key rows decoded into two stages with the 128-byte swizzle;
//   warps 5-7   the same for value rows (rows past the tile's last query and of
//               pages outside the pool are zeros);
//   warps 8-11  head A, 12-15 head B: first their queries, then the online
//               softmax, one thread per query row and all 128 columns; the exponent
//               base moves only when a value passes it by more than 8.  They
//               take over registers from the others.
//
// Every wait is bounded (ptx.cuh); a CTA one of whose waits gave up ends.
#include <math.h>
#include <stddef.h>

#include <algorithm>
#include <type_traits>

#include "attn_plan.cuh"
#include "paged.cuh"

namespace moe {
namespace {

using namespace tc;

constexpr int kPfRows = 128;
constexpr int kPfThreads = 16 * 32;
constexpr int kPfDecWarps = 3;  // that decode keys (warps 2-4), and values (5-7)
constexpr int kPfHeadWarp = 8;                     // first softmax warp
// registers a thread: 512 x 128 at the launch, then two warpgroups each of
// these (2 x 80 + 2 x 176 = 4 x 128)
constexpr int kPfRegsFeed = 80, kPfRegsSoftmax = 176;
static_assert(kPfRegsFeed + kPfRegsSoftmax == 2 * 128, "the launch's registers");
constexpr uint32_t kPfHalf = kPfRows * 128;  // 64 columns of a tile: 16 KB
constexpr uint32_t kPfTile = 2 * kPfHalf;
constexpr uint32_t kPfOffQ = 0;
constexpr uint32_t kPfOffK = 2 * kPfTile;
constexpr uint32_t kPfOffV = 4 * kPfTile;
constexpr uint32_t kPfRaw = kPfRows * kPagedDh;  // a tile as the pages hold it: 16 KB
constexpr uint32_t kPfOffRawK = 6 * kPfTile;
constexpr uint32_t kPfOffRawV = kPfOffRawK + kPfRaw;
constexpr uint32_t kPfOffHdr = kPfOffRawV + kPfRaw;
constexpr uint32_t kPfHdrBytes = 2048;
constexpr size_t kPfSmem = 1024 + kPfOffHdr + kPfHdrBytes;
static_assert(kPfSmem <= 227 * 1024, "shared memory");
// kind::f16: fp16 A and B, fp32 D, M = N = 128; and with B MN-major (bit 16)
constexpr uint32_t kPfIdesc = (1u << 4) | ((uint32_t)(kPfRows >> 3) << 17) | ((uint32_t)(kPfRows >> 4) << 24);
constexpr uint32_t kPfIdescV = kPfIdesc | (1u << 16);
constexpr uint32_t kPfTmemCols = 512, kPfColS = 0, kPfColO = 256;
// probabilities are 2^kPfTop at the exponent base, at most 2^15 where it lags,
// and keep their 11 bits down to 2^-21 of it (2^-32 in the end)
constexpr float kPfTop = 7.f, kPfSlack = 8.f;
constexpr float kPfNone = -1e30f;
constexpr float kPfLeast = 7.888609052210118e-31f;  // 2^-100: nothing times a score
// What row sums are multiplied with: a weight under a value scale of 2^-100 counts as
// up to 2^115 there (2^15 where the base lags), and 2^29 of them stay in range so.
constexpr float kPfSum = 7.62939453125e-6f;  // 2^-17
constexpr int kPfMaxParts = 16, kPfMinTiles = 6;  // of a unit; of a part
constexpr int kPfRing = 8;  // tiles' scales

struct PfScales {
    // of 16 positions each: the key page's scale, log2 and reciprocal (times
    // kPfSum) of the value page's
    float ks[8], lv[8], iv[8];
    // bit i: positions 16 i .. of a page inside the pool; and of one whose keys',
    // values' scale is not zero
    unsigned ok, keys, values;
    int pad[5];
};

struct PfHeader {
    uint64_t q_full[2];    // a head's queries written (four warps)
    uint64_t k_full[2], k_empty[2];
    uint64_t v_full[2], v_empty[2];
    uint64_t t_full[kPfRing];  // a tile's scales written
    uint64_t raw_full[2], raw_empty[2];  // keys', values' rows landed; read by their warps
    // per slot (a head's of two, else a tile's by turns): S written, P, P V finished
    uint64_t s_full[2], p_ready[2], o_full[2];
    uint64_t done;
    uint32_t tmem_base;
    int next;
    int gave_up;
    int last[2];  // a head's part was counted last
    uint32_t nan_rows[kPfRows / 32];  // bit p: NaN among the values of position p0 + p
    alignas(16) PfScales sc[kPfRing];
};
constexpr int kPfBars = (int)((offsetof(PfHeader, done) - offsetof(PfHeader, q_full)) / 8) + 1;
constexpr int pf_bar(size_t off) { return (int)((off - offsetof(PfHeader, q_full)) / 8); }
constexpr int kPfBarP = pf_bar(offsetof(PfHeader, p_ready));
constexpr int kPfBarKF = pf_bar(offsetof(PfHeader, k_full));
constexpr int kPfBarRaw = pf_bar(offsetof(PfHeader, raw_empty));
constexpr int kPfBarVF = pf_bar(offsetof(PfHeader, v_full));
static_assert(sizeof(PfHeader) <= kPfHdrBytes, "header");

__device__ __forceinline__ bool pf_wait(uint64_t *bar, uint32_t parity, unsigned *err) {
    return ptx::mbar_try_wait(bar, parity) || ptx::mbar_wait_hint(bar, parity, err);
}
// a whole warp's
__device__ __forceinline__ bool pf_wait_all(uint64_t *bar, uint32_t parity, unsigned *err) {
    return __all_sync(0xffffffffu, pf_wait(bar, parity, err));
}

__device__ __forceinline__ float pf_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Barrier over head x's softmax threads that also tells whether any of them had p.
__device__ __forceinline__ bool pf_any(int x, bool p) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)p), "r"(1 + x)
        : "memory");
    return r != 0;
}

__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Shared-memory descriptors, 128-byte swizzle, 8 rows 1024 bytes apart: their upper
// half, and the lower one's fields beside the address: K-major, and MN-major with
// the next 64 elements 16 KB on.
constexpr uint32_t kPfDescHi = (1024 >> 4) | 1u << 14 | 2u << 29;
constexpr uint32_t kPfDescK = 1u << 16, kPfDescMn = (kPfHalf >> 4) << 16;

// One lane of the warp, always the same.
__device__ __forceinline__ bool pf_elect() {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r));
    return r != 0;
}

__device__ __forceinline__ void pf_issue_qk(uint32_t d, uint32_t q, uint32_t k) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t at = (i >> 2) * (kPfHalf >> 4) + (i & 3) * 2;
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
            "mov.b64 a, {%1, %4};\n\tmov.b64 b, {%2, %4};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d),
            "r"(q + at), "r"(k + at), "r"(kPfIdesc), "r"(kPfDescHi), "r"(i != 0 ? 1u : 0u)
            : "memory");
    }
}
__device__ __forceinline__ void pf_issue_pv(uint32_t d, uint32_t p_tmem, uint32_t v, uint32_t add) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
            "mov.b64 b, {%2, %4};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d),
            "r"(p_tmem + i * 8), "r"(v + i * (16 * 128 >> 4)), "r"(kPfIdescV), "r"(kPfDescHi),
            "r"(i != 0 ? 1u : add)
            : "memory");
}

__device__ __forceinline__ void pf_tmem_st32(uint32_t taddr, const uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
        "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]),
        "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]),
        "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]),
        "r"(v[29]), "r"(v[30]), "r"(v[31])
        : "memory");
}
__device__ __forceinline__ void pf_tmem_st_wait() {
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

struct PfArgs {
    CUtensorMap tmK, tmV;
    int Hq, Hkv;
    PageView pv;
    AttnPlan plan;
    const bf16 *q;
    const uint8_t *vp;
    const float *ks, *vs;
    bf16 *ctx;
    float *part;  // kPagedUnitParts parts
    int *count;   // of finished parts, a (unit, head of it) each; zero at the start
    unsigned *err;
};

struct PfUnit {
    int t0, rows, p0, sq;  // the tile: first token, tokens, position, sequence
    int g, h0, nh;         // key/value head, first query head, heads
    int j0, n_kv;          // first position tile, position tiles
    int parts, slot0, c;   // its parts, the first one's slot, which one this is
};

// Every tile's pages by TMA, as they are, keys and values each into one buffer
// that its decoding warps empty, and the tile's scales.  A lane a page.  False:
// a wait gave up.
__device__ __forceinline__ bool pf_fetch(const PfArgs &a, PfHeader *hd, unsigned char *smem,
                                         const PfUnit &u) {
    const int lane = threadIdx.x & 31;
    const int shift = a.pv.shift, per = kPfRows >> shift;
    const int last = u.p0 + u.rows - 1;
    const uint64_t pol = ptx::policy_evict_last();
    const int32_t *table = a.pv.table + (size_t)u.sq * a.pv.max_pages;
    auto entry = [&](int j) {
        const int p = (u.j0 + j) * kPfRows + (lane << shift);
        return j < u.n_kv && lane < per && p <= last ? table[p >> shift] : -1;
    };
    int next = entry(0);
    bool good = true;
    int asked[2] = {0, 0};  // tiles
#pragma unroll 1
    for (int j = 0; j < u.n_kv; ++j) {
        const int pg = next >= 0 && next < a.pv.n_pages ? next : -1;
        if (pg < 0 && lane < per && (u.j0 + j) * kPfRows + (lane << shift) <= last)
            set_error(a.err, kErrIndex);
        next = entry(j + 1);
        // the scales of 16 positions a lane
        const int mine = __shfl_sync(0xffffffffu, pg, ((lane & 7) << 4) >> shift);
        float ks = 0.f, vs = 0.f;
        if (mine >= 0 && lane < 8) {
            ks = __ldg(a.ks + (size_t)mine * a.Hkv + u.g);
            vs = __ldg(a.vs + (size_t)mine * a.Hkv + u.g);
        }
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, pg >= 0)) *
                               ((uint32_t)kPagedDh << shift);
        const int row = (pg * a.Hkv + u.g) << shift;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            good = good && pf_wait_all(&hd->raw_empty[v], (uint32_t)(j & 1) ^ 1u, a.err);
            if (!good) break;
            if (lane == 0) ptx::mbar_arrive_expect_tx(&hd->raw_full[v], bytes);
            __syncwarp();
            if (pg >= 0)
                ptx::tma_load_2d(smem + (v ? kPfOffRawV : kPfOffRawK) +
                                     ((uint32_t)(lane * kPagedDh) << shift),
                                 v ? &a.tmV : &a.tmK, 0, row, &hd->raw_full[v], pol);
            ++asked[v];
        }
        PfScales *s = &hd->sc[j % kPfRing];
        if (lane < 8) {
            // (a scale of zero leaves rows of zeros, whatever it counts for here)
            s->ks[lane] = ks;
            s->lv[lane] = log2f(fmaxf(vs, kPfLeast));
            s->iv[lane] = kPfSum / fmaxf(vs, kPfLeast);
        }
        const unsigned ok = __ballot_sync(0xffffffffu, lane < 8 && mine >= 0);
        const unsigned with_keys = __ballot_sync(0xffffffffu, lane < 8 && mine >= 0 && ks != 0.f);
        const unsigned with_values = __ballot_sync(0xffffffffu, lane < 8 && mine >= 0 && vs != 0.f);
        if (lane == 0) {
            s->ok = ok;
            s->keys = with_keys;
            s->values = with_values;
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&hd->t_full[j % kPfRing]);
        if (!good) break;
    }
    // what was asked for lands before the block can exit, also where only the
    // warps that decode it have given up
#pragma unroll
    for (int v = 0; v < 2; ++v)
        if (asked[v] > 0)
            good = pf_wait_all(&hd->raw_full[v], (uint32_t)(asked[v] - 1) & 1u, a.err) && good;
    return good;
}

// A value row that only the tile's rows from p on may see: 0 x NaN is NaN, so its
// NaN become zeros for the product, and pf_show_nan puts them where they belong.
__device__ __forceinline__ void pf_hide_nan(PfHeader *hd, int p, uint4 &x) {
    constexpr uint32_t m = 0x7f7f7f7fu;
    const uint32_t n[4] = {__vcmpeq4(x.x & m, m), __vcmpeq4(x.y & m, m), __vcmpeq4(x.z & m, m),
                           __vcmpeq4(x.w & m, m)};
    if ((n[0] | n[1] | n[2] | n[3]) == 0) return;
    x = make_uint4(x.x & ~n[0], x.y & ~n[1], x.z & ~n[2], x.w & ~n[3]);
    atomicOr(&hd->nan_rows[p >> 5], 1u << (p & 31));
}

// Row r of what has been stored, NaN where a hidden one lies at a position that the
// row sees: dim c at dst + c * step.
template <typename T>
__device__ __noinline__ void pf_show_nan(const PfArgs &a, const PfHeader *hd, const PfUnit &u, int r,
                                         T *dst, int step) {
    for (int w = 0; w <= r >> 5; ++w)
        for (uint32_t m = hd->nan_rows[w]; m; m &= m - 1) {
            const int p = w * 32 + __ffs(m) - 1;
            if (p > r) return;
            const int pos = u.p0 + p, pg = a.pv.page(u.sq, pos >> a.pv.shift);
            const uint8_t *row = a.vp + ((((size_t)pg * a.Hkv + u.g) << a.pv.shift) +
                                         (pos & ((1 << a.pv.shift) - 1))) * kPagedDh;
            for (int c = 0; c < kPagedDh; ++c)
                if ((row[c] & 0x7f) == 0x7f) dst[c * step] = from_f<T>(__uint_as_float(0x7fffffffu));
        }
}
__device__ __forceinline__ bool pf_any_nan(const PfHeader *hd) {
    return (hd->nan_rows[0] | hd->nan_rows[1] | hd->nan_rows[2] | hd->nan_rows[3]) != 0;
}

// 16 e4m3 numbers -> fp16, as chunks 2c, 2c + 1 of a row of 64 dims.
__device__ __forceinline__ void pf_decode16(const uint4 &x, unsigned char *d0, unsigned char *d1) {
    const uint32_t v[4] = {x.x, x.y, x.z, x.w};
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[2 * i] = e4m3x2_to_f16x2(v[i] & 0xffffu);
        y[2 * i + 1] = e4m3x2_to_f16x2(v[i] >> 16);
    }
    *reinterpret_cast<uint4 *>(d0) = make_uint4(y[0], y[1], y[2], y[3]);
    *reinterpret_cast<uint4 *>(d1) = make_uint4(y[4], y[5], y[6], y[7]);
}

// A tile's rows decoded into one operand's two stages, four rows (a quarter warp
// each) a time of warp w of three, every third four of them.  These warps' issue
// slots are what the kernel has least of, so a tile whose rows every query sees
// takes nothing but a load, the conversions and two stores at offsets that a lane
// forms once (checks in the same loop: 512 tokens at position 5000 163 us, 115 so).
// False: a wait gave up.
__device__ __forceinline__ bool pf_decode(const PfArgs &a, PfHeader *hd, unsigned char *smem,
                                          const PfUnit &u, bool keys, int w) {
    constexpr int B = 6;                                   // fours of rows a batch
    constexpr int N = (kPfRows / 4 + kPfDecWarps - 1) / kPfDecWarps;  // two batches of N at most
    const int lane = threadIdx.x & 31;
    const int last = u.p0 + u.rows - 1;
    uint64_t *full = keys ? hd->k_full : hd->v_full, *empty = keys ? hd->k_empty : hd->v_empty;
    uint64_t *raw_full = &hd->raw_full[keys ? 0 : 1], *raw_empty = &hd->raw_empty[keys ? 0 : 1];
    const unsigned char *raw = smem + (keys ? kPfOffRawK : kPfOffRawV) + w * 512 + lane * 16;
    // row 4 f + lane / 8, dims 16 (lane % 8) ..: its chunks in the 64-dim half's row,
    // in fours f of even and of odd distance from w
    const uint32_t row0 = w * 4 + (lane >> 3), c = (lane & 3) * 2;
    unsigned char *dst = smem + (keys ? kPfOffK : kPfOffV) + ((lane & 7) >> 2) * kPfHalf + row0 * 128;
    const uint32_t e0 = (c ^ (row0 & 7)) << 4, e1 = ((c + 1) ^ (row0 & 7)) << 4;
    const uint32_t o0 = e0 ^ 64u, o1 = e1 ^ 64u;  // (4 rows on: bit 2 of the row)
#pragma unroll 1
    for (int j = 0; j < u.n_kv; ++j) {
        const int b = j & 1;
        if (!pf_wait_all(&hd->t_full[j % kPfRing], (uint32_t)(j / kPfRing) & 1u, a.err) ||
            !pf_wait_all(raw_full, j & 1, a.err) ||
            !pf_wait_all(&empty[b], ((uint32_t)(j >> 1) & 1u) ^ 1u, a.err))
            return false;
        // rows that hold no position are zeros, as are those under a scale of zero
        const unsigned ok = keys ? hd->sc[j % kPfRing].keys : hd->sc[j % kPfRing].values;
        const int at = (u.j0 + j) * kPfRows;
        unsigned char *d = dst + b * kPfTile;
        auto rows = [&](auto check) {
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                uint4 x[B];
#pragma unroll
                for (int k = 0; k < B; ++k) {
                    const int n = half * B + k;
                    if (k < N - B - 1 || w + n * kPfDecWarps < kPfRows / 4)
                        x[k] = *reinterpret_cast<const uint4 *>(raw + n * kPfDecWarps * 512);
                }
                if (half == 1) {
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(raw_empty);
                }
#pragma unroll
                for (int k = 0; k < B; ++k) {
                    const int n = half * B + k;
                    if (!(k < N - B - 1 || w + n * kPfDecWarps < kPfRows / 4)) continue;
                    if constexpr (decltype(check)::value) {
                        const int row = row0 + n * kPfDecWarps * 4;
                        if (at + row > last || !((ok >> (row >> 4)) & 1u))
                            x[k] = make_uint4(0u, 0u, 0u, 0u);
                        if (!keys && at + row > u.p0) pf_hide_nan(hd, at + row - u.p0, x[k]);
                    }
                    pf_decode16(x[k], d + n * kPfDecWarps * 512 + (k & 1 ? o0 : e0),
                                d + n * kPfDecWarps * 512 + (k & 1 ? o1 : e1));
                }
            }
        };
        if (ok == 0xffu && at + kPfRows - 1 <= (keys ? last : u.p0))
            rows(std::false_type());
        else
            rows(std::true_type());
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&full[b]);
    }
    return true;
}
static_assert(kPfDecWarps % 2 == 1 /* and B even */, "the fours of a warp alternate in their rows' bit 2");

// The MMA issuer's part of a unit: P_k V_k, then S of the tile after next for one
// head, which has two places (slots) for S and P and its softmax no pause, or of the
// next for two, each of which has one place and works while the other's products
// run.  S replaces P only after P V has finished.  (Two places of 64 positions each for
// two heads: products of N = 64 take as long as those of 128, 133 us for 512 tokens
// at position 5000 instead of 94.  P V of 64 positions at a time, as soon as their P is
// there: the warp waits for the second half instead of starting the other head's,
// 98.)
//
// The whole warp runs it and one lane issues: operands that are the same in every
// lane by the code go to the uniform registers that the instructions take them from
// at once.  A branch of one lane's moves each there first, 85 cycles an instruction
// of 64: 117 us.  False: a wait gave up.
__device__ __forceinline__ bool pf_issue(PfHeader *hd, uint32_t sbase, const PfUnit &u,
                                         unsigned *err) {
    const int n = __shfl_sync(0xffffffffu, u.n_kv, 0), nh = __shfl_sync(0xffffffffu, u.nh, 0);
    const uint32_t tmem = __shfl_sync(0xffffffffu, hd->tmem_base, 0);
    const uint32_t q0 = ((sbase + kPfOffQ) >> 4) | kPfDescK, k0 = ((sbase + kPfOffK) >> 4) | kPfDescK;
    const uint32_t v0 = ((sbase + kPfOffV) >> 4) | kPfDescMn;
    const bool lead = pf_elect();
    auto slot = [&](int x, int k) { return nh == 2 ? x : k & 1; };
    auto phase = [&](int k) { return (uint32_t)(nh == 2 ? k : k >> 1) & 1u; };
    const int ahead = 3 - nh;  // of S
#pragma unroll 1
    for (int k = -ahead; k < n; ++k)
#pragma unroll 1
        for (int x = 0; x < nh; ++x) {
            if (k >= 0) {
                const int b = k & 1, s = slot(x, k);
                if (x == 0 && !pf_wait_all(&hd->v_full[b], (uint32_t)(k >> 1) & 1u, err)) return false;
                if (!pf_wait_all(&hd->p_ready[s], phase(k), err)) return false;
                tc_fence_after();
                if (lead) {
                    pf_issue_pv(tmem + kPfColO + x * 128, tmem + kPfColS + s * 128, v0 + b * (kPfTile >> 4), k != 0);
                    mma_commit(&hd->o_full[s]);
                    if (x == nh - 1) mma_commit(&hd->v_empty[b]);
                }
                __syncwarp();
            }
            const int i = k + ahead;
            if (i < n) {
                const int b = i & 1, s = slot(x, i);
                if (i == 0 && !pf_wait_all(&hd->q_full[x], 0, err)) return false;
                if (x == 0 && !pf_wait_all(&hd->k_full[b], (uint32_t)(i >> 1) & 1u, err)) return false;
                if (k >= 0 && !pf_wait_all(&hd->o_full[s], phase(k), err)) return false;
                tc_fence_after();
                if (lead) {
                    pf_issue_qk(tmem + kPfColS + s * 128, q0 + x * (kPfTile >> 4), k0 + b * (kPfTile >> 4));
                    mma_commit(&hd->s_full[s]);
                    if (x == nh - 1) mma_commit(&hd->k_empty[b]);
                }
                __syncwarp();
            }
        }
    return true;
}

// Head x's queries, scaled to fp16 in shared memory, by the head's four warps: 32
// rows a warp, two of them (16 lanes each) at a time.  What row r's scores are to
// be multiplied with, r the thread's.  (A row a thread, 16 loads of 32 lines each,
// kept the first tiles' loads waiting, and pf_store's stores alike: a prompt of 1000
// tokens 39.0 us, 33.5 with both so.)
__device__ __forceinline__ float pf_queries(const PfArgs &a, unsigned char *smem, const PfUnit &u,
                                            int x, int r) {
    const int lane = r & 31, r0 = r - lane, half = lane >> 4, c = lane & 15;
    const uint4 *src = reinterpret_cast<const uint4 *>(
                           a.q + ((size_t)u.t0 * a.Hq + u.h0 + x) * kPagedDh) + c;
    const size_t step = (size_t)a.Hq * (kPagedDh / 8);
    uint4 w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int row = r0 + 2 * i + half;
        w[i] = row < u.rows ? src[row * step] : make_uint4(0u, 0u, 0u, 0u);
    }
    // a row's largest magnitude, as bf16; rows of i and i + 8 side by side
    uint32_t m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t p[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint4 v = w[i + 8 * k];
            p[k] = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu),
                            __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
        }
        m[i] = __vmaxu2(__byte_perm(p[0], p[1], 0x5410), __byte_perm(p[0], p[1], 0x7632));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m[i] = __vmaxu2(m[i], __shfl_xor_sync(0xffffffffu, m[i], o));
    }
    unsigned char *q = smem + kPfOffQ + x * kPfTile + (c >> 3) * kPfHalf;
    uint32_t mine = 0;  // the thread's own row's
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t mb = i < 8 ? m[i] & 0xffffu : m[i - 8] >> 16;
        const int e = min(max((int)(mb >> 7), 15), 254);
        // (a row with NaN or an infinity: NaN)
        const float up = __uint_as_float(mb < 0x7f80u ? (uint32_t)(254 + 14 - e) << 23 : 0x7fffffffu);
        const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
        uint32_t y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float lo, hi;
            unpack_bf16x2(v[k], lo, hi);
            y[k] = f16x2(lo * up, hi * up);
        }
        const int row = r0 + 2 * i + half;
        *reinterpret_cast<uint4 *>(q + row * 128 + (((c & 7) ^ (row & 7)) << 4)) =
            make_uint4(y[0], y[1], y[2], y[3]);
        const uint32_t of = __shfl_sync(0xffffffffu, (uint32_t)e, (lane & 1) << 4);
        mine = (lane >> 1) == i ? of : mine;
    }
    // log2(e) / sqrt(128)
    return 0.12751743f * __uint_as_float((mine - 14u) << 23);
}

// Rows of head x's O, divided by their sums, to ctx: a row's bf16 go through the
// head's queries' place (no product reads them any more), so that 16 lanes store a
// row.
__device__ __forceinline__ void pf_store(const PfArgs &a, unsigned char *smem, const PfUnit &u,
                                         int x, int r, uint32_t o_col, float l) {
    const int lane = r & 31, r0 = r - lane;
    const float inv = l == 0.f ? 0.f : kPfSum / l;
    unsigned char *s = smem + kPfOffQ + x * kPfTile;
#pragma unroll
    for (int c = 0; c < 128; c += 32) {
        float v[32];
        tmem_ld32(o_col + c, v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 p2 =
                    __floats2bfloat162_rn(v[i + 2 * e] * inv, v[i + 2 * e + 1] * inv);
                w[e] = *reinterpret_cast<const uint32_t *>(&p2);
            }
            *reinterpret_cast<uint4 *>(s + r * 256 + ((((c + i) >> 3) ^ (r & 7)) << 4)) =
                make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    __syncwarp();
    const int ch = lane & 15;
    bf16 *dst = a.ctx + ((size_t)u.t0 * a.Hq + u.h0 + x) * kPagedDh + ch * 8;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int row = r0 + 2 * i + (lane >> 4);
        if (row < u.rows)
            *reinterpret_cast<uint4 *>(dst + (size_t)row * a.Hq * kPagedDh) =
                *reinterpret_cast<const uint4 *>(s + row * 256 + ((ch ^ (row & 7)) << 4));
    }
    __syncwarp();  // (before pf_show_nan, and the next unit's queries)
}

// One row's softmax over a unit's tiles; m, l: its exponent base, its sum.
__device__ __forceinline__ bool pf_softmax(PfHeader *hd, uint32_t s_cols, uint32_t o_col,
                                           const PfUnit &u, int r, int x, float qs, float &m,
                                           float &l, unsigned *err) {
    const int lane = threadIdx.x & 31;
    m = kPfNone;
    l = 0.f;
    bool good = true;
#pragma unroll 1
    for (int j = 0; j < u.n_kv; ++j) {
        const int slot = u.nh == 2 ? x : j & 1;
        const uint32_t phase = (uint32_t)(u.nh == 2 ? j : j >> 1) & 1u, s_col = s_cols + slot * 128;
        const int lim = u.p0 + r - (u.j0 + j) * kPfRows;  // the row's last position in the tile
        good = good && pf_wait_all(&hd->t_full[j % kPfRing], (uint32_t)(j / kPfRing) & 1u, err);
        good = good && pf_wait_all(&hd->s_full[slot], phase, err);
        tc_fence_after();
        float v[128];
#pragma unroll
        for (int c = 0; c < 128; c += 32)
            tmem_ld32(s_col + c, *reinterpret_cast<float(*)[32]>(&v[c]));
        tmem_ld_wait();
        const PfScales *sc = &hd->sc[j % kPfRing];
        const unsigned ok = sc->ok;
        float cs[8], lv[8];
        *reinterpret_cast<float4 *>(&cs[0]) = *reinterpret_cast<const float4 *>(&sc->ks[0]);
        *reinterpret_cast<float4 *>(&cs[4]) = *reinterpret_cast<const float4 *>(&sc->ks[4]);
        *reinterpret_cast<float4 *>(&lv[0]) = *reinterpret_cast<const float4 *>(&sc->lv[0]);
        *reinterpret_cast<float4 *>(&lv[4]) = *reinterpret_cast<const float4 *>(&sc->lv[4]);
        if ((u.j0 + j) * kPfRows + kPfRows - 1 > u.p0 || ok != 0xffu) {
            // positions past the row's own, and without a page: their score is
            // -inf (cs is positive)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int n = (ok >> i) & 1u ? lim - 16 * i : -1;
#pragma unroll
                for (int k = 0; k < 16; ++k)
                    if (k > n) v[16 * i + k] = -INFINITY;
            }
        }
        float mrow = kPfNone;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float m2[2] = {v[16 * i], v[16 * i + 1]};
#pragma unroll
            for (int k = 2; k < 16; ++k) m2[k & 1] = fmaxf(m2[k & 1], v[16 * i + k]);
            cs[i] = fmaxf(cs[i] * qs, kPfLeast);
            mrow = fmaxf(mrow, fmaf(fmaxf(m2[0], m2[1]), cs[i], lv[i]));
        }
        const bool bump = mrow > m + kPfSlack;
        const float corr = bump ? pf_exp2(m - mrow) : 1.f;
        if (bump) m = mrow;
        const bool rescale = __any_sync(0xffffffffu, bump) && j >= 1 && good;
        float lt = 0.f;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t pw[32];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int gi = half * 4 + i;
                // p vs: the value page's scale is part of the exponent; the row
                // sum takes it out again
                const float b = lv[gi] + (kPfTop - m);
                const float2 c2 = make_float2(cs[gi], cs[gi]), b2 = make_float2(b, b);
                float2 sum2[2];
#pragma unroll
                for (int k = 0; k < 16; k += 2) {
                    const int c = 16 * gi + k;
                    const float2 e = __ffma2_rn(make_float2(v[c], v[c + 1]), c2, b2);
                    const float2 w = make_float2(pf_exp2(e.x), pf_exp2(e.y));
                    sum2[(k >> 1) & 1] = k < 4 ? w : __fadd2_rn(sum2[(k >> 1) & 1], w);
                    pw[i * 8 + (k >> 1)] = f16x2(w.x, w.y);
                }
                lt = fmaf((sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y), sc->iv[gi], lt);
            }
            pf_tmem_st32(s_col + half * 32, pw);
        }
        // a new base rescales O: P_{j-1} V_{j-1} finished before S_j was issued,
        // and P_j V_j waits for this warp's arrival
        if (rescale) {
            // (one head's S_j is issued ahead of P_{j-1} V_{j-1})
            if (u.nh == 1)
                good = pf_wait_all(&hd->o_full[slot ^ 1], (uint32_t)((j - 1) >> 1) & 1u, err);
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 128; c += 32) {
                float ov[32];
                uint32_t ow[32];
                tmem_ld32(o_col + c, ov);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) ow[i] = __float_as_uint(ov[i] * corr);
                pf_tmem_st32(o_col + c, ow);
            }
        }
        pf_tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&hd->p_ready[slot]);
        l = l * corr + lt;
    }
    return good;
}

// Unit `unit` of S parts of each (tile, heads).
__device__ __forceinline__ PfUnit pf_unit(const PfArgs &a, int unit, int G, int per, bool single,
                                          int S) {
    PfUnit u;
    const int whole = unit / S;
    u.c = unit - whole * S;
    u.slot0 = whole * S;
    const int tile = whole / (a.Hkv * per), gp = whole - tile * a.Hkv * per;
    const int4 td = __ldcg(&a.plan.tiles[tile]);
    u.g = gp / per;
    const int hp = gp - u.g * per;
    u.h0 = u.g * G + (single ? hp : 2 * hp);
    u.nh = !single && 2 * hp + 1 < G ? 2 : 1;
    u.t0 = td.x;
    u.rows = td.y;
    u.p0 = td.z;
    u.sq = td.w;
    const int n = (u.p0 + u.rows - 1) / kPfRows + 1;
    u.parts = min(S, n);
    // (a unit of fewer tiles than parts has nothing for the last ones)
    u.j0 = u.c < u.parts ? (int)((long long)u.c * n / u.parts) : n;
    u.n_kv = u.c < u.parts ? (int)((long long)(u.c + 1) * n / u.parts) - u.j0 : 0;
    return u;
}

// A part of a head's rows left in the workspace, a column's rows side by side;
// the part that is counted last merges them all.  Thread r its row.
__device__ __noinline__ void pf_part(const PfArgs &a, PfHeader *hd, const PfUnit &u, int x, int r,
                                        uint32_t o_col, float m, float l) {
    constexpr size_t kHead = (size_t)kPfRows * (128 + 2);  // a head's part
    auto at = [&](int c) { return a.part + ((size_t)(u.slot0 + c) * 2 + x) * kHead; };
    float *mine = at(u.c);
#pragma unroll 1
    for (int c = 0; c < 128; c += 32) {
        float v[32];
        tmem_ld32(o_col + c, v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 32; ++i) mine[(c + i) * kPfRows + r] = v[i];
    }
    if (pf_any_nan(hd)) pf_show_nan(a, hd, u, r, mine + r, kPfRows);
    reinterpret_cast<float2 *>(mine + 128 * kPfRows)[r] = make_float2(m, l);
    auto meet = [&]() { pf_any(x, false); };  // the head's threads
    meet();
    if (r == 0) {
        __threadfence();
        hd->last[x] = atomicAdd(&a.count[u.slot0 * 2 + x], 1) == u.parts - 1;
        __threadfence();
    }
    meet();
    if (!hd->last[x] || r >= u.rows) return;
    float M = kPfNone, L = 0.f;
    {
        float2 ml[kPfMaxParts];
#pragma unroll
        for (int c = 0; c < kPfMaxParts; ++c)
            ml[c] = __ldcg(reinterpret_cast<const float2 *>(at(min(c, u.parts - 1)) + 128 * kPfRows) + r);
#pragma unroll
        for (int c = 0; c < kPfMaxParts; ++c) M = fmaxf(M, ml[c].x);
#pragma unroll
        for (int c = 0; c < kPfMaxParts; ++c)
            L = c < u.parts ? fmaf(pf_exp2(ml[c].x - M), ml[c].y, L) : L;
    }
    const float inv = L == 0.f ? 0.f : kPfSum / L;
    bf16 *dst = a.ctx + ((size_t)(u.t0 + r) * a.Hq + u.h0 + x) * kPagedDh;
    // (64 columns' loads go out together: with eight 20 us for three parts)
#pragma unroll 1
    for (int c0 = 0; c0 < 128; c0 += 64) {
        float s[64];
#pragma unroll
        for (int i = 0; i < 64; ++i) s[i] = 0.f;
#pragma unroll 1
        for (int c = 0; c < u.parts; ++c) {
            const float *p = at(c) + c0 * kPfRows + r;
            const float2 ml = __ldcg(reinterpret_cast<const float2 *>(at(c) + 128 * kPfRows) + r);
            float v[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) v[i] = __ldcg(p + i * kPfRows);
            const float w = pf_exp2(ml.x - M);
#pragma unroll
            for (int i = 0; i < 64; ++i) s[i] = fmaf(w, v[i], s[i]);
        }
#pragma unroll
        for (int i = 0; i < 64; i += 8) {
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 p2 =
                    __floats2bfloat162_rn(s[i + 2 * e] * inv, s[i + 2 * e + 1] * inv);
                o[e] = *reinterpret_cast<const uint32_t *>(&p2);
            }
            *reinterpret_cast<uint4 *>(dst + c0 + i) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

__global__ void __launch_bounds__(kPfThreads, 1)
k_paged_prefill_tc(const __grid_constant__ PfArgs a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    PfHeader *hd = reinterpret_cast<PfHeader *>(smem + kPfOffHdr);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = a.Hq / a.Hkv, pairs = (G + 1) / 2;
    const uint32_t sbase = ptx::smem_u32(smem);
    unsigned *err = a.err;

    // ahead of the wait: what needs nothing of the plan
    if (threadIdx.x == 0) {
        hd->gave_up = 0;
        ptx::prefetch_tmap(&a.tmK);
        ptx::prefetch_tmap(&a.tmV);
    }
    if (warp == 0) tmem_alloc(&hd->tmem_base, kPfTmemCols);
    // the barriers of a unit, before and after the block meets
    auto begin = [&](bool again) {
        if (threadIdx.x < kPfBars) {
            const int i = threadIdx.x;
            if (again) ptx::mbar_inval(hd->q_full + i);
            // (q_full and p_ready: a head's four warps; k_full, v_full and
            // raw_empty: the decoding ones)
            auto of = [&](int first, int n) { return i >= first && i < first + n; };
            ptx::mbar_init(hd->q_full + i, of(0, 2) || of(kPfBarP, 2) ? 4
                                           : of(kPfBarKF, 2) || of(kPfBarVF, 2) || of(kPfBarRaw, 2)
                                               ? kPfDecWarps
                                               : 1);
            ptx::fence_barrier_init();
        }
        if (threadIdx.x < kPfRows / 32) hd->nan_rows[threadIdx.x] = 0u;
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    };
    begin(false);
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    const int n_tiles = __ldcg(&a.plan.head->n_tiles);
    const int4 longest = __ldcg(&a.plan.tiles[0]);  // (read whether there is one or not)
    // Two heads a unit or one, and a unit whole or, where there are at least two CTAs
    // to each, cut along the positions into up to kPfMaxParts parts of kPfMinTiles
    // tiles or more: whichever ends first for units as long as the longest, counting
    // 1.85 us for a position tile of two heads, 1.3 of one, 5 us to start and leave a
    // unit, and 8 and 1 for each part where they are merged (measured: 512 tokens at
    // position 5000, 44 tiles, 4 x 48 heads on 152 SMs, 94 us in pairs, 133 alone).
    // A lane a choice.
    // (the plan's last bin holds tiles of any length from there on, in any order, and
    // the choice decides what is added first)
    const int n_long = n_tiles > 0 ? min((longest.z + longest.y - 1) / kPfRows + 1, kPlanBins) : 1;
    bool single;
    int S;
    {
        const bool one = lane & 2, whole = !(lane & 1);
        const int units = max(1, n_tiles * a.Hkv * (one ? G : pairs)), cost = one ? 26 : 37;
        const int most = min(min(kPfMaxParts, (int)gridDim.x / units), n_long / kPfMinTiles);
        const int parts = whole ? 1 : max(most, 1);
        const int rounds = (units * parts + (int)gridDim.x - 1) / (int)gridDim.x;
        const long long us20 = (long long)rounds * ((n_long + parts - 1) / parts * cost + 100) +
                               (whole ? 0 : 160 + 20 * parts);
        const unsigned key = (unsigned)min(us20, (1LL << 29) - 1) << 2 | (lane & 3);
        const unsigned best = __reduce_min_sync(0xffffffffu, whole || most > 1 ? key : 0xffffffffu);
        single = best & 2;
        S = __shfl_sync(0xffffffffu, parts, best & 3);
    }
    const int per = single ? G : pairs;
    const int n_whole = n_tiles * a.Hkv * per;
    const int n_units = n_whole * S;
    int unit = (int)blockIdx.x;
    if (unit >= n_units) {
        if (warp == 0) tmem_dealloc(hd->tmem_base, kPfTmemCols);
        return;
    }
    // the next unit, for all, its barriers made; false: there is none
    auto more = [&]() {
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        unit = hd->next;
        if (unit >= n_units || hd->gave_up) return false;
        begin(true);  // (meets: all have read what the next unit writes)
        return true;
    };

    if (warp < kPfHeadWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPfRegsFeed));
#pragma unroll 1
        do {
            const PfUnit u = pf_unit(a, unit, G, per, single, S);
            bool good = true;
            if (warp == 0) {
                if (u.n_kv > 0) {
                    good = pf_issue(hd, sbase, u, err);
                    if (pf_elect()) mma_commit(&hd->done);
                    good &= pf_wait_all(&hd->done, 0, err);
                    // the MMAs' last arrivals, before the barriers start anew
                    for (int j = max(0, u.n_kv - 2); good && j < u.n_kv; ++j)
                        good = pf_wait_all(&hd->k_empty[j & 1], (uint32_t)(j >> 1) & 1u, err) &&
                               pf_wait_all(&hd->v_empty[j & 1], (uint32_t)(j >> 1) & 1u, err);
                }
            } else if (warp == 1) {
                good = pf_fetch(a, hd, smem, u);
                if (lane == 0) hd->next = (int)gridDim.x + atomicAdd(&a.plan.head->next, 1);
            } else {
                const bool keys = warp < 2 + kPfDecWarps;
                good = pf_decode(a, hd, smem, u, keys, warp - (keys ? 2 : 2 + kPfDecWarps));
            }
            if (!good) hd->gave_up = 1;
        } while (more());
        if (warp == 0) tmem_dealloc(hd->tmem_base, kPfTmemCols);
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPfRegsSoftmax));
        const int x = (warp - kPfHeadWarp) / 4;
        const int q = warp & 3, r = q * 32 + lane;
#pragma unroll 1
        do {
            const PfUnit u = pf_unit(a, unit, G, per, single, S);
            if (x < u.nh && u.n_kv > 0) {
                const uint32_t at = hd->tmem_base + ((uint32_t)(q * 32) << 16);
                const uint32_t o_col = at + kPfColO + x * 128;
                const float qs = pf_queries(a, smem, u, x, r);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&hd->q_full[x]);
                float m = kPfNone, l = 0.f;
                bool good = pf_softmax(hd, at + kPfColS, o_col, u, r, x, qs, m, l, err);
                good = good && pf_wait_all(&hd->o_full[u.nh == 2 ? x : (u.n_kv - 1) & 1],
                                           (uint32_t)(u.nh == 2 ? u.n_kv - 1 : (u.n_kv - 1) >> 1) & 1u, err);
                if (!good) hd->gave_up = 1;
                // (the head's warps meet in pf_part: one that gave up, none goes there)
                if (u.parts > 1 && pf_any(x, !good)) good = false;
                if (good) tc_fence_after();
                if (good && u.parts > 1) {
                    pf_part(a, hd, u, x, r, o_col, m, l);
                } else if (good) {
                    pf_store(a, smem, u, x, r, o_col, l);
                    if (pf_any_nan(hd) && r < u.rows)
                        pf_show_nan(a, hd, u, r,
                                    a.ctx + ((size_t)(u.t0 + r) * a.Hq + u.h0 + x) * kPagedDh, 1);
                }
            }
        } while (more());
    }
}

}  // namespace

cudaError_t launch_paged_prefill_tc(const PagedAttn &a, const AttnPlan &plan, float *part,
                                    int *count, cudaStream_t st) {
    const void *kern = (const void *)k_paged_prefill_tc;
    static SmemOnce once;
    cudaError_t e = once.set(kern, kPfSmem);
    if (e != cudaSuccess) return e;
    PfArgs pa{{}, {}, a.Hq, a.Hkv, a.pv, plan, static_cast<const bf16 *>(a.q),
              static_cast<const uint8_t *>(a.vp), a.ks, a.vs, static_cast<bf16 *>(a.ctx), part,
              count, device_info().err};
    if (!paged_map(&pa.tmK, a.kp, a, false) || !paged_map(&pa.tmV, a.vp, a, false))
        return cudaErrorInvalidValue;
    void *args[] = {&pa};
    const int ctas = std::min(device_info().sm_count, kPagedUnitParts);
    const long long most = (long long)kPfMaxParts * a.Hq * (a.T / kPagedTileMinRows);
    LaunchScope ls("paged_prefill_tc", st);
    return launch_pdl(
        kern, dim3((unsigned)std::max(1LL, std::min<long long>(most, ctas))),
        dim3(kPfThreads), kPfSmem, st, args);
}

}  // namespace moe
