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
// Each k-block is an accumulator of its own in tensor memory (4 of them in turn): the
// epilogue multiplies it with the block's scales as it adds it to the sum it keeps in
// registers.  Warp 0 loads (TMA), warp 1 issues the MMAs, warps 2-5 are the epilogue, thread i
// of lane quarter q = (128 weight rows) row 32 q + i.
#include "quant.cuh"

namespace moe {
namespace {

using namespace tc;

constexpr int kQsThreads = 192;
constexpr int kQsAcc = 4;           // accumulators in tensor memory
constexpr int kQsMinBlocks = 4;     // k-blocks of a CTA's share at least
constexpr int kQsMaxStages = 12;
constexpr uint32_t kQsTile = 128 * 128;

struct QsHeader {
    uint64_t full[kQsMaxStages], empty[kQsMaxStages];
    uint64_t tfull[kQsAcc], tempty[kQsAcc];
    uint64_t done;
    uint32_t tmem_base;
    int last;
    int prefix[257];       // tiles of the experts ahead
    alignas(16) float scale[2][2][64];  // of this k-block: x's times w1's (w's), times v1's
    uint32_t amax[4][64];
};
constexpr uint32_t kQsHdrBytes = 4096;
static_assert(sizeof(QsHeader) <= kQsHdrBytes, "header");

template <bool UP, int N>
struct QsCfg {
    static constexpr int kMats = UP ? 2 : 1;
    static constexpr uint32_t kStage = kMats * kQsTile + N * 128;
    static constexpr int kStages = (int)((200 * 1024) / kStage) < kQsMaxStages ? (int)((200 * 1024) / kStage)
                                                                              : kQsMaxStages;
    static constexpr size_t kSmem = 1024 + kStages * kStage + kQsHdrBytes;
    static constexpr uint32_t kCols = kMats * N;  // tensor-memory columns of an accumulator
    static constexpr uint32_t kTmem = kQsAcc * kCols < 32 ? 32 : kQsAcc * kCols;
    // kind::f8f6f4: e4m3 A and B, fp32 D, both K-major, M = 128
    static constexpr uint32_t kIdesc = (1u << 4) | ((128u >> 4) << 24) | ((uint32_t)(N >> 3) << 17);
    static_assert(kStage % 1024 == 0, "stages stay 1024-byte aligned");
    static_assert(kSmem <= 227 * 1024, "shared memory");
    static_assert((kTmem & (kTmem - 1)) == 0 && kTmem <= 512, "tensor memory");
};

__device__ __forceinline__ void tma_3d(void *dst, const CUtensorMap *m, int32_t x, int32_t y,
                                       int32_t z, uint64_t *bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        ".L2::cache_hint [%0], [%1, {%2, %3, %4}], [%5], %6;" ::"r"(ptx::smem_u32(dst)),
        "l"(m), "r"(x), "r"(y), "r"(z), "r"(ptx::smem_u32(bar)), "l"(policy)
        : "memory");
}

__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
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
    long long W, pos, end;
    int ctas, cta;

    __device__ __forceinline__ void start(int n_ctas, int me) {
        W = (long long)prefix[E] * nk;
        ctas = (int)max(1LL, min((long long)n_ctas, W / kQsMinBlocks));
        cta = me;
        pos = me < ctas ? W * me / ctas : W;
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

// prefix[e]: tiles of the experts ahead of e.
__device__ void qs_prefix(const int32_t *offsets, int E, int S, int nwt, int cols, int *prefix,
                          unsigned *err) {
    const int lane = threadIdx.x & 31;
    int run = 0;
    for (int base = 0; base < E; base += 32) {
        const int e = base + lane;
        int c = 0;
        if (e < E) {
            const int lo = offsets ? offsets[e] : 0, hi = offsets ? offsets[e + 1] : S;
            if (lo < 0 || hi < lo || hi > S) set_error(err, kErrIndex);
            else c = ((hi - lo + cols - 1) / cols) * nwt;
        }
        int incl = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (e < E) prefix[e] = run + incl - c;
        run += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) prefix[E] = run;
}

struct QsArgs {
    const int32_t *offsets;
    int E, S, n_in, n_out;
    const float *xs, *s0, *s1;  // scales of x [blocks, S], of w1 (or w), of v1
    void *out;                  // h8 or y
    float *out_scale;           // hs [blocks, S]
    int y_bf16;
    float *part;
    int *count;
    unsigned *err;
};

template <bool UP, int N>
__global__ void __launch_bounds__(kQsThreads, 1)
k_quant_stream(const __grid_constant__ CUtensorMap tm_w0, const __grid_constant__ CUtensorMap tm_w1,
               const __grid_constant__ CUtensorMap tm_x, const QsArgs a) {
    using C = QsCfg<UP, N>;
    constexpr int kStages = C::kStages;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    QsHeader *hd = reinterpret_cast<QsHeader *>(smem + kStages * C::kStage);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nk = q_blocks(a.n_in), nwt = q_blocks(a.n_out);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(&hd->full[s], 1);
            ptx::mbar_init(&hd->empty[s], 1);
        }
        for (int b = 0; b < kQsAcc; ++b) {
            ptx::mbar_init(&hd->tfull[b], 1);
            ptx::mbar_init(&hd->tempty[b], 4);
        }
        ptx::mbar_init(&hd->done, 1);
        ptx::fence_barrier_init();
        ptx::prefetch_tmap(&tm_w0);
        if (UP) ptx::prefetch_tmap(&tm_w1);
        ptx::prefetch_tmap(&tm_x);
    }
    if (warp == 1) tmem_alloc(&hd->tmem_base, C::kTmem);
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    if (warp == 2) qs_prefix(a.offsets, a.E, a.S, nwt, N, hd->prefix, a.err);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = hd->tmem_base;
    QsShare share{hd->prefix, a.offsets, a.E, a.S, nk, N};
    share.start((int)gridDim.x, (int)blockIdx.x);
    QsTile t;
    int kb0, kb1, first, last;

    if (warp == 0) {
        // ------------------------------------------------------------ loads
        if (lane == 0) {
            const uint64_t pol_w = ptx::policy_evict_first(), pol_x = ptx::policy_evict_last();
            uint32_t it = 0;
            bool ok = true;
            while (ok && share.next(t, kb0, kb1, first, last)) {
                for (int kb = kb0; kb < kb1; ++kb, ++it) {
                    const uint32_t s = it % kStages, ph = (it / kStages) & 1;
                    if (!(ok = wait_soon(&hd->empty[s], ph ^ 1, a.err))) break;
                    unsigned char *sp = smem + s * C::kStage;
                    ptx::mbar_arrive_expect_tx(&hd->full[s], C::kStage);
                    tma_3d(sp, &tm_w0, kb * 128, t.wt * 128, t.e, &hd->full[s], pol_w);
                    if (UP) tma_3d(sp + kQsTile, &tm_w1, kb * 128, t.wt * 128, t.e, &hd->full[s], pol_w);
                    ptx::tma_load_2d(sp + C::kMats * kQsTile, &tm_x, kb * 128, t.s0, &hd->full[s],
                                     pol_x);
                }
            }
            // copies in flight land before the block can end
            for (uint32_t k = (it > kStages ? it - kStages : 0); k < it; ++k)
                ptx::mbar_wait_hint(&hd->full[k % kStages], (k / kStages) & 1, a.err);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMAs
        const bool one = elect_one();
        uint32_t it = 0;
        bool ok = true;
        while (ok && share.next(t, kb0, kb1, first, last)) {
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const uint32_t s = it % kStages, ph = (it / kStages) & 1;
                const uint32_t b = it % kQsAcc, bph = (it / kQsAcc) & 1;
                ok = wait_soon(&hd->full[s], ph, a.err) &&
                     wait_soon(&hd->tempty[b], bph ^ 1, a.err);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t sa = ptx::smem_u32(smem + s * C::kStage);
                const uint64_t w0 = smem_desc(sa), w1 = smem_desc(sa + kQsTile);
                const uint64_t x = smem_desc(sa + C::kMats * kQsTile);
                const uint32_t d = tmem + b * C::kCols;
                if (one) {
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) {
                        mma_f8(d, w0 + 2 * kk, x + 2 * kk, C::kIdesc, kk != 0);
                        if (UP) mma_f8(d + N, w1 + 2 * kk, x + 2 * kk, C::kIdesc, kk != 0);
                    }
                    mma_commit(&hd->empty[s]);
                    mma_commit(&hd->tfull[b]);
                }
                __syncwarp();
            }
        }
        if (one) {
            mma_commit(&hd->done);
            ptx::mbar_wait(&hd->done, 0, a.err);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ epilogue
        const int q = warp & 3, th = q * 32 + lane;  // row of the weight tile
        bool dead = false;  // a wait gave up: keep the barriers, skip the work
        uint32_t it = 0;
        while (share.next(t, kb0, kb1, first, last)) {
            float acc[C::kMats][N];
#pragma unroll
            for (int m = 0; m < C::kMats; ++m)
#pragma unroll
                for (int i = 0; i < N; ++i) acc[m][i] = 0.f;
            const float *sw0 = a.s0 + ((size_t)t.e * nwt + t.wt) * nk;
            const float *sw1 = UP ? a.s1 + ((size_t)t.e * nwt + t.wt) * nk : nullptr;
            const float *sx = a.xs + t.s0 + th;
            const bool mine = th < t.cnt;
            float nx = mine ? sx[(size_t)kb0 * a.S] : 0.f, n0 = sw0[kb0], n1 = UP ? sw1[kb0] : 0.f;
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const uint32_t b = it % kQsAcc, bph = (it / kQsAcc) & 1;
                if (th < N) {
                    hd->scale[it & 1][0][th] = nx * n0;
                    if (UP) hd->scale[it & 1][1][th] = nx * n1;
                }
                if (kb + 1 < kb1) {
                    nx = mine ? sx[(size_t)(kb + 1) * a.S] : 0.f;
                    n0 = sw0[kb + 1];
                    if (UP) n1 = sw1[kb + 1];
                }
                ptx::named_bar_sync(1, 128);
                if (!dead) dead = !__all_sync(0xffffffffu, wait_soon(&hd->tfull[b], bph, a.err));
                tc_fence_after();
                const uint32_t base = tmem + ((uint32_t)(q * 32) << 16) + b * C::kCols;
#pragma unroll
                for (int m = 0; m < C::kMats; ++m)
#pragma unroll
                    for (int c = 0; c < N; c += 16) {
                        float v[16];
                        if (!dead) {
                            tmem_ld16(base + m * N + c, v);
                            tmem_ld_wait();
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i) v[i] = 0.f;
                        }
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const float4 sc = *reinterpret_cast<const float4 *>(&hd->scale[it & 1][m][c + i]);
                            acc[m][c + i] = fmaf(sc.x, v[i], acc[m][c + i]);
                            acc[m][c + i + 1] = fmaf(sc.y, v[i + 1], acc[m][c + i + 1]);
                            acc[m][c + i + 2] = fmaf(sc.z, v[i + 2], acc[m][c + i + 2]);
                            acc[m][c + i + 3] = fmaf(sc.w, v[i + 3], acc[m][c + i + 3]);
                        }
                    }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&hd->tempty[b]);
            }
            if (first != last) {
                // this piece into its slot: a CTA's last piece may begin a tile that the next
                // ones end, its others end or continue one
                constexpr size_t kSlot = (size_t)C::kMats * N * 128;
                float *mine_p = a.part + (size_t)(2 * share.cta + (kb0 == 0 ? 1 : 0)) * kSlot + th;
#pragma unroll
                for (int m = 0; m < C::kMats; ++m)
#pragma unroll
                    for (int i = 0; i < N; ++i) mine_p[(m * N + i) * 128] = acc[m][i];
                __threadfence();
                ptx::named_bar_sync(1, 128);
                if (th == 0) hd->last = atomicAdd(a.count + first, 1) == last - first;
                ptx::named_bar_sync(1, 128);
                if (!hd->last) continue;
                __threadfence();
#pragma unroll
                for (int m = 0; m < C::kMats; ++m)
#pragma unroll
                    for (int i = 0; i < N; ++i) acc[m][i] = 0.f;
                for (int c = first; c <= last; ++c) {
                    const float *p = a.part + (size_t)(2 * c + (c == first ? 1 : 0)) * kSlot + th;
#pragma unroll
                    for (int m = 0; m < C::kMats; ++m)
#pragma unroll
                        for (int i = 0; i < N; ++i) acc[m][i] += __ldcg(p + (m * N + i) * 128);
                }
            }
            const int row = t.wt * 128 + th;
            if (UP) {
                // h in place of a; its largest magnitude of each column over the 128 rows
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    acc[0][i] = q_silu(acc[0][i]) * acc[C::kMats - 1][i];
                    const uint32_t m = __reduce_max_sync(0xffffffffu, abs_bits(acc[0][i]));
                    if (lane == 0) hd->amax[q][i] = m;
                }
                ptx::named_bar_sync(1, 128);
                uint8_t *h = static_cast<uint8_t *>(a.out) + (size_t)t.s0 * a.n_out + row;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (i < t.cnt) {
                        const uint32_t m = max(max(hd->amax[0][i], hd->amax[1][i]),
                                               max(hd->amax[2][i], hd->amax[3][i]));
                        float sc, inv;
                        q_scale(m, sc, inv);
                        if (row < a.n_out && !dead)
                            h[(size_t)i * a.n_out] = (uint8_t)e4m3x2(acc[0][i] * inv, 0.f);
                        if (th == i && !dead) a.out_scale[(size_t)t.wt * a.S + t.s0 + i] = sc;
                    }
                }
            } else if (row < a.n_out && !dead) {
                if (a.y_bf16) {
                    bf16 *y = static_cast<bf16 *>(a.out) + (size_t)t.s0 * a.n_out + row;
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (i < t.cnt) y[(size_t)i * a.n_out] = __float2bfloat16_rn(acc[0][i]);
                } else {
                    float *y = static_cast<float *>(a.out) + (size_t)t.s0 * a.n_out + row;
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (i < t.cnt) y[(size_t)i * a.n_out] = acc[0][i];
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
cudaError_t launch(const QuantGemm &g, const void *w0, const void *w1, QsArgs a, cudaStream_t st) {
    using C = QsCfg<UP, N>;
    CUtensorMap mw0, mw1, mx;
    if (!q_weight_map(&mw0, w0, g.E, g.n_out, g.n_in) ||
        !q_weight_map(&mw1, UP ? w1 : w0, g.E, g.n_out, g.n_in) ||
        !q_row_map(&mx, g.x8, g.S, g.n_in, N))
        return cudaErrorInvalidValue;
    const void *kern = (const void *)k_quant_stream<UP, N>;
    static SmemOnce smem;
    cudaError_t e = smem.set(kern, C::kSmem);
    if (e != cudaSuccess) return e;
    a.offsets = g.offsets;
    a.E = g.E;
    a.S = g.S;
    a.n_in = g.n_in;
    a.n_out = g.n_out;
    a.xs = g.xs;
    a.err = device_info().err;
    void *args[] = {&mw0, &mw1, &mx, &a};
    LaunchScope ls(UP ? "quant_up_stream" : "quant_down_stream", st);
    return launch_pdl(kern, dim3(std::min(device_info().sm_count, kQMaxCtas)), dim3(kQsThreads),
                      C::kSmem, st, args);
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
    if (cols == 16) return launch<true, 16>(g, u.w1, u.v1, a, st);
    if (cols == 32) return launch<true, 32>(g, u.w1, u.v1, a, st);
    return launch<true, 64>(g, u.w1, u.v1, a, st);
}

cudaError_t launch_quant_stream_down(const QuantGemm &g, const QuantDown &u, const QuantParts &p,
                                     int cols, cudaStream_t st) {
    QsArgs a{};
    a.s0 = u.s;
    a.out = u.y;
    a.y_bf16 = u.y_bf16;
    a.part = p.part;
    a.count = p.count;
    if (cols == 16) return launch<false, 16>(g, u.w, nullptr, a, st);
    if (cols == 32) return launch<false, 32>(g, u.w, nullptr, a, st);
    return launch<false, 64>(g, u.w, nullptr, a, st);
}

}  // namespace moe
