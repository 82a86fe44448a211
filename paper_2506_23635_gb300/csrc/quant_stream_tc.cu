// Grouped products of 8-bit operands for few rows a group: the weights stream through
// the SMs once, as the MMA's M operand, the rows of a group as its N (16, 32 or 64).
//
//   DOWN:  y[j, n] = sum_b xs[j, b] ws[e, n/128, b] (sum_{k in block b} x8[j, k] w8[e, n, k])
//   UP:    a, b = the same with w1 and v1;  h = SiLU(a) b, quantised in blocks of 128
//
// Bound by the weights' bytes.  All tiles (expert, 128 weight rows, run of rows) times
// k-blocks of 128 are one line of work that the CTAs, one on each SM, share out
// equally; a tile that several CTAs have a piece of is added up by the one that finishes
// last, in the order of the k-blocks whoever that is.
//
// Each k-block is an accumulator of its own in tensor memory (a few in turn): the
// epilogue multiplies it with the block's scales as it adds it to the sum it keeps in
// registers.  Up to 32 columns, two sets of epilogue warps take the k-blocks in turn (one set
// alone took about as long for a k-block as its weights take from memory) and are added at a
// piece's end; of 64 columns each set has half.  Warp 0 loads (TMA), warp 1 issues the MMAs,
// the others are the epilogue: thread i of a warp of lane quarter q has weight row 32 q + i.
//
// Measured: 16 rows of 38912 x 16384 100 us, 6.4 TB/s of weights (0.94 of a copy's rate); one row
// of 8192 x 6144 14 us with the launch ahead (7.4 at the copy's rate); 16 experts of
// 6144 x 10752, 16 rows each, up 314 us and down 159 (0.99 and 0.98); 40 of 2000 x 1424 with 30
// rows each (64 columns) 63 and 43 us, the epilogue's.
#include "quant.cuh"

namespace moe {
namespace {

using namespace tc;

constexpr int kQsMinBlocks = 4;     // k-blocks of a CTA's share at least
constexpr int kQsMaxStages = 12;
constexpr uint32_t kQsTile = 128 * 128;

constexpr uint32_t kQsHdrBytes = 7168;
struct QsHeader {
    uint64_t full[kQsMaxStages], empty[kQsMaxStages];
    uint64_t tfull[4], tempty[4];
    uint64_t done;
    uint32_t tmem_base;
    int last, ready[2];  // (ready: of the shared piece that ends or continues a tile, that begins one)
    int prefix[257];       // tiles of the experts ahead
    alignas(16) float scale[8][2][2][32];  // warp, k-blocks in turn: x's times w1's (w's), v1's
    uint32_t amax[4][64];
    alignas(16) float hinv[64];  // (UP) one over the scales of h's columns
};
static_assert(sizeof(QsHeader) <= kQsHdrBytes, "header");

template <bool UP, int N>
struct QsCfg {
    static constexpr int kMats = UP ? 2 : 1;
    static constexpr uint32_t kStage = kMats * kQsTile + N * 128;
    // eight epilogue warps: two sets that take the k-blocks in turn, with 64 columns two
    // halves of them
    static constexpr int kSets = N == 64 ? 1 : 2, kThreads = 64 + 256;
    static constexpr int kOwn = N == 64 ? 32 : N;  // columns of a warp
    // the second set's sums on their way to the first
    static constexpr uint32_t kSums = kSets == 2 ? kMats * N * 512 : 0;
    // With 16 columns the up and the down projection's CTAs share an SM, so that the down
    // projection's first weights arrive during the up projection's end (wider tiles take too many
    // registers); alone: as many stages as fit.
    static constexpr int kShared = N != 16 ? 0 : UP ? 3 : 4;
    static constexpr int kFit = (int)((220 * 1024 - kSums - kQsHdrBytes) / kStage);
    static constexpr int kAlone = kFit < kQsMaxStages ? kFit : kQsMaxStages;
    static constexpr int kAcc = 4;  // accumulators in turn
    static constexpr uint32_t kCols = kMats * N;  // tensor-memory columns of an accumulator
    static constexpr uint32_t kTmem = kAcc * kCols;
    // kind::f8f6f4: e4m3 A and B, fp32 D, both K-major, M = 128
    static constexpr uint32_t kIdesc = (1u << 4) | ((128u >> 4) << 24) | ((uint32_t)(N >> 3) << 17);
    static constexpr size_t smem(int stages) { return 1024 + stages * kStage + kSums + kQsHdrBytes; }
    static_assert(kStage % 1024 == 0, "stages stay 1024-byte aligned");
    static_assert(smem(kAlone) <= 227 * 1024, "shared memory");
    static_assert((kTmem & (kTmem - 1)) == 0 && kTmem >= 32 && kTmem <= 512, "tensor memory");
};
static_assert(QsCfg<true, 16>::smem(QsCfg<true, 16>::kShared) + QsCfg<false, 16>::smem(QsCfg<false, 16>::kShared) <= 226 * 1024,
              "an up and a down projection's CTA on one SM");

__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ int load_acquire(const int *p) {
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ int add_acq_rel(int *p, int v) {
    int r;
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], %2;" : "=r"(r) : "l"(p), "r"(v) : "memory");
    return r;
}

__device__ __forceinline__ void bar_arrive(uint32_t id, uint32_t threads) {
    asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

struct QsTile {
    int e, wt;    // expert, 128 weight rows
    int s0, cnt;  // first row of x, rows
};

// A CTA's share of the line of work: pieces of tiles.
struct QsShare {
    const int *prefix;
    const int32_t *offsets;
    int E, S, nk, cols;
    long long W, begin, pos, end;
    int ctas, cta;

    __device__ __forceinline__ void start(int n_ctas, int me) {
        W = (long long)prefix[E] * nk;
        ctas = (int)max(1LL, min((long long)n_ctas, W / kQsMinBlocks));
        cta = me;
        begin = pos = me < ctas ? W * me / ctas : W;
        end = me < ctas ? W * (me + 1) / ctas : W;
    }
    __device__ __forceinline__ int owner(long long block) const {
        return (int)(((block + 1) * ctas - 1) / W);
    }
    // the next piece: k-blocks [kb0, kb1) of tile t; CTAs first..last have a piece of it
    __device__ __forceinline__ bool next(QsTile &t, int &kb0, int &kb1, int &first, int &last) {
        if (pos >= end) return false;
        const int u = (int)(pos / nk);
        const long long b0 = (long long)u * nk;
        kb0 = (int)(pos - b0);
        kb1 = (int)min((long long)nk, end - b0);
        pos = b0 + kb1;
        first = kb0 == 0 ? cta : owner(b0);
        last = kb1 == nk ? cta : owner(b0 + nk - 1);
        t.e = chunk_expert(prefix, E, u);
        const int lo = offsets ? offsets[t.e] : 0, hi = offsets ? offsets[t.e + 1] : S;
        const int nst = (hi - lo + cols - 1) / cols, r = u - prefix[t.e];
        t.wt = r / nst;
        const int st = r - t.wt * nst;
        t.s0 = lo + st * cols;
        t.cnt = min(cols, hi - t.s0);
        return true;
    }
};

struct QsArgs {
    const int32_t *offsets;
    int E, S, n_in, n_out;
    const float *xs, *s0, *s1;  // scales of x [blocks, S], of w1 (or w), of v1
    void *out;                  // h8 or y
    float *out_scale;           // hs [blocks, S]
    int y_bf16;
    int stages;
    float *part;
    int *count;
    unsigned *err;
};

template <bool UP, int N>
__global__ void __launch_bounds__(QsCfg<UP, N>::kThreads, N == 16 ? 2 : 1)
k_quant_stream(const __grid_constant__ CUtensorMap tm_w0, const __grid_constant__ CUtensorMap tm_w1,
               const __grid_constant__ CUtensorMap tm_x, const QsArgs a) {
    using C = QsCfg<UP, N>;
    constexpr int kAcc = C::kAcc;
    const int n_stage = a.stages;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    QsHeader *hd = reinterpret_cast<QsHeader *>(smem + n_stage * C::kStage + C::kSums);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nk = q_blocks(a.n_in), nwt = q_blocks(a.n_out);
    if (threadIdx.x == 0) {
        for (int s = 0; s < n_stage; ++s) {
            ptx::mbar_init(&hd->full[s], 1);
            ptx::mbar_init(&hd->empty[s], 1);
        }
        for (int b = 0; b < kAcc; ++b) {
            ptx::mbar_init(&hd->tfull[b], 1);
            ptx::mbar_init(&hd->tempty[b], 8 / C::kSets);
        }
        ptx::mbar_init(&hd->done, 1);
        ptx::fence_barrier_init();
        ptx::prefetch_tmap(&tm_w0);
        if (UP) ptx::prefetch_tmap(&tm_w1);
        ptx::prefetch_tmap(&tm_x);
    }
    if (warp == 1) tmem_alloc(&hd->tmem_base, C::kTmem);
    ptx::launch_dependents();
    // (the offsets are older than the launch ahead, which lets this one start behind its own
    // wait only, or is started so itself)
    if (warp == 2) q_tile_prefix(a.offsets, a.E, a.S, nwt, N, hd->prefix, a.err);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = hd->tmem_base;
    QsShare share{hd->prefix, a.offsets, a.E, a.S, nk, N};
    share.start((int)gridDim.x, (int)blockIdx.x);
    QsTile t{};
    int kb0, kb1, first, last;

    if (warp == 0) {
        // ------------------------------------------------------------ loads
        if (lane == 0) {
            const uint64_t pol_w = ptx::policy_evict_first(), pol_x = ptx::policy_evict_last();
            auto weights = [&](int s, int kb) {
                unsigned char *sp = smem + s * C::kStage;
                ptx::mbar_arrive_expect_tx(&hd->full[s], C::kStage);
                tma_3d(sp, &tm_w0, kb * 128, t.wt * 128, t.e, &hd->full[s], pol_w);
                if (UP) tma_3d(sp + kQsTile, &tm_w1, kb * 128, t.wt * 128, t.e, &hd->full[s], pol_w);
            };
            // the first stages' weights, which no kernel ahead writes, before the wait
            int early = 0;
            for (QsShare peek = share; early < n_stage && peek.next(t, kb0, kb1, first, last);)
                for (int kb = kb0; kb < kb1 && early < n_stage; ++kb, ++early) weights(early, kb);
            ptx::grid_dependency_wait();
            int s = 0, n = 0;
            uint32_t ph = 1;
            bool ok = true;
            while (ok && share.next(t, kb0, kb1, first, last)) {
                for (int kb = kb0; kb < kb1; ++kb, ++n) {
                    if (!(ok = wait_soon(&hd->empty[s], ph, a.err))) break;
                    if (n >= early) weights(s, kb);
                    ptx::tma_load_2d(smem + s * C::kStage + C::kMats * kQsTile, &tm_x, kb * 128, t.s0,
                                     &hd->full[s], pol_x);
                    if (++s == n_stage) {
                        s = 0;
                        ph ^= 1;
                    }
                }
            }
            // copies in flight land before the block can end: the stages that were filled
            // last, whose barriers' phases are those of their last fills.  (Where a wait
            // gave up, stages whose weights came early may wait for rows that do not come:
            // these waits end too.)
            const int total = max(n, early);
            for (int k = max(0, total - n_stage); k < total; ++k)
                ptx::mbar_wait_hint(&hd->full[k % n_stage], (k / n_stage) & 1, a.err);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMAs
        const bool one = elect_one();
        const uint64_t d0 = smem_desc(ptx::smem_u32(smem));
        int s = 0;
        uint32_t ph = 0;
        bool ok = true;
#pragma unroll 1
        for (uint32_t it = 0, n = (uint32_t)(share.end - share.pos); ok && it < n; ++it) {
            const uint32_t b = it % kAcc, bph = (it / kAcc) & 1;
            ok = wait_soon(&hd->full[s], ph, a.err) && wait_soon(&hd->tempty[b], bph ^ 1, a.err);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const uint64_t w0 = d0 + s * (C::kStage >> 4), w1 = w0 + (kQsTile >> 4);
            const uint64_t x = w0 + C::kMats * (kQsTile >> 4);
            const uint32_t d = tmem + b * C::kCols;
            if (one) {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                    mma_f8(d, w0 + 2 * kk, x + 2 * kk, C::kIdesc, kk != 0);
                    if (UP) mma_f8(d + N, w1 + 2 * kk, x + 2 * kk, C::kIdesc, kk != 0);
                }
                mma_commit(&hd->tfull[b]);
                mma_commit(&hd->empty[s]);
            }
            __syncwarp();
            if (++s == n_stage) {
                s = 0;
                ph ^= 1;
            }
        }
        if (one) {
            mma_commit(&hd->done);
            ptx::mbar_wait(&hd->done, 0, a.err);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ epilogue
        // th: row of the weight tile; columns c0 .. c0 + kOwn; et: thread of the set
        constexpr int kOwn = C::kOwn, kSets = C::kSets, kEt = 256 / kSets;
        const int q = warp & 3, th = q * 32 + lane;
        const int set = kSets == 2 ? (warp - 2) >> 2 : 0, half = kSets == 2 ? 0 : (warp - 2) >> 2;
        const int c0 = half * kOwn, et = half * 128 + th;
        float(*scale)[2][32] = hd->scale[warp - 2];
        float *sums = reinterpret_cast<float *>(smem + n_stage * C::kStage) + c0 * 128 + th;
        bool dead = false;  // a wait gave up: keep the barriers, skip the work
        uint32_t it = 0, piece = 0, turn = 0;
        ptx::grid_dependency_wait();  // (x's scales; the result's last readers)
        for (; share.next(t, kb0, kb1, first, last); ++piece) {
            uint64_t sum[C::kMats][kOwn / 2];  // two columns each
#pragma unroll
            for (int m = 0; m < C::kMats; ++m)
#pragma unroll
                for (int i = 0; i < kOwn / 2; ++i) sum[m][i] = 0;
            const float *sw0 = a.s0 + ((size_t)t.e * nwt + t.wt) * nk;
            const float *sw1 = UP ? a.s1 + ((size_t)t.e * nwt + t.wt) * nk : nullptr;
            // lane i: column c0 + i's scale (lanes behind the last row: the first row's, which count for nothing)
            const bool mine = lane < kOwn && c0 + lane < t.cnt;
            const float *sx = a.xs + t.s0 + (mine ? c0 + lane : 0);
            int kb = kb0;
            if (kSets == 2 && ((it ^ set) & 1)) {
                ++kb;
                ++it;
            }
            float nx = 0.f, n0 = 0.f, n1 = 0.f;
            if (kb < kb1) {
                nx = sx[(size_t)kb * a.S];
                n0 = sw0[kb];
                if (UP) n1 = sw1[kb];
            }
            for (; kb < kb1; kb += kSets, it += kSets, turn ^= 1) {
                const uint32_t b = it % kAcc, bph = (it / kAcc) & 1;
                if (lane < kOwn) {
                    scale[turn][0][lane] = nx * n0;
                    if (UP) scale[turn][1][lane] = nx * n1;
                }
                if (kb + kSets < kb1) {
                    nx = sx[(size_t)(kb + kSets) * a.S];
                    n0 = sw0[kb + kSets];
                    if (UP) n1 = sw1[kb + kSets];
                }
                if (!dead) dead = !__all_sync(0xffffffffu, wait_soon(&hd->tfull[b], bph, a.err));
                __syncwarp();
                tc_fence_after();
                const uint32_t base = tmem + ((uint32_t)(q * 32) << 16) + b * C::kCols + c0;
                if (!dead) {
#pragma unroll
                    for (int m = 0; m < C::kMats; ++m) {
                        float v[kOwn];
                        if constexpr (kOwn == 16) tmem_ld16(base + m * N, v);
                        else tmem_ld32(base + m * N, v);
                        tmem_ld_wait();
                        if (m == C::kMats - 1) {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) ptx::mbar_arrive(&hd->tempty[b]);
                        }
                        const ulonglong2 *sc = reinterpret_cast<const ulonglong2 *>(scale[turn][m]);
#pragma unroll
                        for (int i = 0; i < kOwn / 4; ++i) {
                            const ulonglong2 f = sc[i];
                            fma2(sum[m][2 * i], v[4 * i], v[4 * i + 1], f.x);
                            fma2(sum[m][2 * i + 1], v[4 * i + 2], v[4 * i + 3], f.y);
                        }
                    }
                }
            }
            it = (uint32_t)(share.pos - share.begin);  // k-blocks of the share so far
            if (set == 1) {  // its sums to the first set
                if (piece) ptx::named_bar_sync(2, 2 * kEt);  // (the last ones are read)
#pragma unroll
                for (int m = 0; m < C::kMats; ++m)
#pragma unroll
                    for (int i = 0; i < kOwn / 2; ++i) {
                        const float2 f = both(sum[m][i]);
                        sums[(m * N + 2 * i) * 128] = f.x;
                        sums[(m * N + 2 * i + 1) * 128] = f.y;
                    }
                bar_arrive(1, 2 * kEt);
                continue;
            }
            // are the tile's other pieces all done?  (That of its first k-blocks is the last of a
            // CTA's share, the others the first ones of theirs: each has a word of its own, as nothing
            // holds the warps together at the pieces between them.)
            const int begins = kb0 == 0;
            if (first != last && et == 0)
                hd->ready[begins] = load_acquire(a.count + first) == last - first;
            if (kSets == 2) ptx::named_bar_sync(1, 2 * kEt);
            else if (first != last) ptx::named_bar_sync(3, kEt);
            float acc[C::kMats][kOwn];
#pragma unroll
            for (int m = 0; m < C::kMats; ++m)
#pragma unroll
                for (int i = 0; i < kOwn / 2; ++i) {
                    const float2 f = both(sum[m][i]);
                    acc[m][2 * i] = f.x;
                    acc[m][2 * i + 1] = f.y;
                    if (kSets == 2) {
                        acc[m][2 * i] += sums[(m * N + 2 * i) * 128];
                        acc[m][2 * i + 1] += sums[(m * N + 2 * i + 1) * 128];
                    }
                }
            if (kSets == 2) bar_arrive(2, 2 * kEt);
            if (first != last) {
                // Slots of pieces: a CTA's last piece may begin a tile that the next ones end, its
                // others end or continue one.
                constexpr size_t kSlot = (size_t)C::kMats * N * 128;
                bool whole = hd->ready[begins];
                if (!whole) {
                    float *to = a.part + (size_t)(2 * share.cta + begins) * kSlot + c0 * 128 + th;
#pragma unroll
                    for (int m = 0; m < C::kMats; ++m)
#pragma unroll
                        for (int i = 0; i < kOwn; ++i) to[(m * N + i) * 128] = acc[m][i];
                    ptx::named_bar_sync(3, kEt);
                    // (the barrier hands this thread the others' writes, its release all of them)
                    if (et == 0) hd->last = add_acq_rel(a.count + first, 1) == last - first;
                    ptx::named_bar_sync(3, kEt);
                    whole = hd->last;
                }
                if (!whole) continue;
                // in the order of the k-blocks, whoever adds: the sums are the same bits
#pragma unroll
                for (int m = 0; m < C::kMats; ++m)
#pragma unroll
                    for (int j = 0; j < kOwn; j += 16) {
                        float all[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) all[i] = 0.f;
                        for (int c = first; c <= last; ++c) {
                            const float *p = a.part + (size_t)(2 * c + (c == first ? 1 : 0)) * kSlot +
                                             (m * N + c0 + j) * 128 + th;
                            const bool me = c == share.cta;
#pragma unroll
                            for (int i = 0; i < 16; ++i) all[i] += me ? acc[m][j + i] : __ldcg(p + i * 128);
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[m][j + i] = all[i];
                    }
            }
            const int row = t.wt * 128 + th;
            if (UP) {
                // h in place of a; its largest magnitude of each column over the 128 rows
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    acc[0][i] = q_silu(acc[0][i]) * acc[C::kMats - 1][i];
                    const uint32_t m = __reduce_max_sync(0xffffffffu, abs_bits(acc[0][i]));
                    if (lane == 0) hd->amax[q][c0 + i] = m;
                }
                ptx::named_bar_sync(3, kEt);
                if (et < N) {
                    const uint32_t m = max(max(hd->amax[0][et], hd->amax[1][et]),
                                           max(hd->amax[2][et], hd->amax[3][et]));
                    float sc, inv;
                    q_scale(m, sc, inv);
                    hd->hinv[et] = inv;
                    if (et < t.cnt && !dead) a.out_scale[(size_t)t.wt * a.S + t.s0 + et] = sc;
                }
                ptx::named_bar_sync(3, kEt);
                uint8_t *h = static_cast<uint8_t *>(a.out) + (size_t)(t.s0 + c0) * a.n_out + row;
                const int left = row < a.n_out && !dead ? t.cnt - c0 : 0;
                const float4 *inv4 = reinterpret_cast<const float4 *>(&hd->hinv[c0]);
#pragma unroll
                for (int i = 0; i < kOwn; i += 4) {
                    const float4 inv = inv4[i / 4];
                    const uint32_t w = e4m3x2(acc[0][i] * inv.x, acc[0][i + 1] * inv.y) |
                                       e4m3x2(acc[0][i + 2] * inv.z, acc[0][i + 3] * inv.w) << 16;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (i + j < left) h[(size_t)(i + j) * a.n_out] = (uint8_t)(w >> (8 * j));
                }
            } else if (row < a.n_out && !dead) {
                if (a.y_bf16) {
                    bf16 *y = static_cast<bf16 *>(a.out) + (size_t)(t.s0 + c0) * a.n_out + row;
#pragma unroll
                    for (int i = 0; i < kOwn; ++i)
                        if (c0 + i < t.cnt) y[(size_t)i * a.n_out] = __float2bfloat16_rn(acc[0][i]);
                } else {
                    float *y = static_cast<float *>(a.out) + (size_t)(t.s0 + c0) * a.n_out + row;
#pragma unroll
                    for (int i = 0; i < kOwn; ++i)
                        if (c0 + i < t.cnt) y[(size_t)i * a.n_out] = acc[0][i];
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, C::kTmem);
}

template <bool UP, int N>
cudaError_t launch(const QuantGemm &g, const void *w0, const void *w1, QsArgs a, bool alone,
                   cudaStream_t st) {
    using C = QsCfg<UP, N>;
    CUtensorMap mw0, mw1, mx;
    if (!q_weight_map(&mw0, w0, g.E, g.n_out, g.n_in) ||
        !q_weight_map(&mw1, UP ? w1 : w0, g.E, g.n_out, g.n_in) ||
        !q_row_map(&mx, g.x8, g.S, g.n_in, N))
        return cudaErrorInvalidValue;
    const void *kern = (const void *)k_quant_stream<UP, N>;
    static SmemOnce smem;
    cudaError_t e = smem.set(kern, C::smem(C::kAlone));
    if (e != cudaSuccess) return e;
    a.offsets = g.offsets;
    a.E = g.E;
    a.S = g.S;
    a.n_in = g.n_in;
    a.n_out = g.n_out;
    a.xs = g.xs;
    a.stages = alone || C::kShared == 0 ? C::kAlone : C::kShared;
    a.err = device_info().err;
    void *args[] = {&mw0, &mw1, &mx, &a};
    LaunchScope ls(UP ? "quant_up_stream" : "quant_down_stream", st);
    return launch_pdl(kern, dim3(std::min(device_info().sm_count, kQMaxCtas)), dim3(C::kThreads),
                      C::smem(a.stages), st, args);
}

}  // namespace

cudaError_t launch_quant_stream_up(const QuantGemm &g, const QuantUp &u, const QuantParts &p,
                                   int cols, cudaStream_t st) {
    QsArgs a{};
    a.s0 = u.s1;
    a.s1 = u.sv;
    a.out = u.h8;
    a.out_scale = u.hs;
    a.part = p.part;
    a.count = p.count;
    if (cols == 16) return launch<true, 16>(g, u.w1, u.v1, a, false, st);
    if (cols == 32) return launch<true, 32>(g, u.w1, u.v1, a, false, st);
    return launch<true, 64>(g, u.w1, u.v1, a, false, st);
}

cudaError_t launch_quant_stream_down(const QuantGemm &g, const QuantDown &u, const QuantParts &p,
                                     int cols, bool alone, cudaStream_t st) {
    QsArgs a{};
    a.s0 = u.s;
    a.out = u.y;
    a.y_bf16 = u.y_bf16;
    a.part = p.part;
    a.count = p.count;
    if (cols == 16) return launch<false, 16>(g, u.w, nullptr, a, alone, st);
    if (cols == 32) return launch<false, 32>(g, u.w, nullptr, a, alone, st);
    return launch<false, 64>(g, u.w, nullptr, a, alone, st);
}

}  // namespace moe
