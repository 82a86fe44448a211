// Grouped products of 8-bit operands for many rows a group: CTAs of 128 rows of x as their MMAs'
// M, 256 weight rows as their N.
//
//   DOWN:  y[j, n] = sum_b xs[j, b] ws[e, n/128, b] (sum_{k in block b} x8[j, k] w8[e, n, k])
//   UP:    a, b = the same with w1 and v1;  h = SiLU(a) b, quantised in blocks of 128
//
// A k-block of 128 is an accumulator of its own (two of 256 columns fill the tensor memory);
// eight epilogue warps take turns with the MMAs, which write one accumulator while the other
// is multiplied with the block's scales and added to the sums in registers.  The rows of x
// are the lanes, so that a thread needs one scale of x times one or two of the weights for
// each k-block: with the weights as lanes every column would need its own, 32 lanes reading
// the same word of shared memory.
//
// Bound by the way around: a k-block takes 0.51 us, about 970 cycles (9728 rows of 8192 x 6144:
// 392 us, 2.5 PFLOP/s), its MMAs 512, what shared memory moves for it (48 KB in, 48 KB out) 750 at
// least, a buffer's sums 580 in the epilogue, and an accumulator goes from one to the other and
// back.  Every CTA loads its weight tile by itself, from L2 where others take the same one.  Pairs of
// CTAs that load half of a tile each for both of them (MMAs of two CTAs, cta_group::2): 388 us,
// but runs of 256 rows, of which short groups fill less.
// Scales of powers of two could go into the MMAs (kind::mxf8f6f4, no epilogue before the end):
// 321 us, but any other scale needs this way, and the choice a look at all scales first.
//
// N: 256 rows of the weights; for UP 128 rows of W1, then the same 128 of V1.  Epilogue warp (q,
// half): lanes 32 q .. and half of the columns (UP: 64 of a and the same 64 of b), 128 sums a thread.
//
// Units are (expert, weight tile, run of 128 rows), runs innermost, so that units that run
// together share weight tiles in L2.  CTA c of C takes units c, c + C, ...
#include "quant.cuh"

namespace moe {
namespace {

using namespace tc;

// warp 0 loads, warp 1 issues the MMAs, warps 2 and 3 prepare scales, warps 4-11 are the
// epilogue.  Registers of the launch: 168 a thread, 64,512; what the first four warps give up the
// others take: 128 (136 + 2 * 184) = 64,512 (splits that spill on either side cost 5 to 20%).
constexpr int kQwThreads = 384;
constexpr int kQwRegsFeed = 136, kQwRegsSums = 184;
constexpr int kQwEpilogue = 4;  // first warp of it
constexpr uint32_t kQwTile = 128 * 128;
constexpr uint32_t kQwStage = 3 * kQwTile;  // 128 rows of x, 256 weight rows
constexpr int kQwMaxStages = 4;
// kind::f8f6f4: e4m3 A and B, fp32 D, both K-major, M = 128, N = 256
constexpr uint32_t kQwIdesc = (1u << 4) | ((256u >> 3) << 17) | ((128u >> 4) << 24);

struct QwHeader {
    uint64_t full[kQwMaxStages], empty[kQwMaxStages];
    uint64_t tfull[2], tempty[2];
    uint64_t done;
    uint32_t tmem_base;
    int prefix[257];
    float2 scale[4][128];      // steps in turn, row: x's times w1's and v1's (the tile's two blocks')
    uint32_t amax[2][2][128];  // (UP) of a row's 64 columns: tile in turn, half
};
constexpr uint32_t kQwHdrBytes = 8192;
static_assert(sizeof(QwHeader) <= kQwHdrBytes, "header");
// y's way out: 4 KB an epilogue warp, 32 rows of 128 bytes.  (h goes out from registers, and
// its projection has a stage more: 1027 -> 1010 us for 2048 tokens; rows of 64 bytes and a stage
// more for y, too, 99 -> 102.)
template <bool UP>
struct QwCfg {
    static constexpr int kStages = UP ? 4 : 3;
    static constexpr uint32_t kOut = UP ? 0 : 8 * 4096;
    static constexpr size_t kSmem = 1024 + kStages * kQwStage + kOut + kQwHdrBytes;
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

// x, w: the lower halves of their descriptors (the upper: 128-byte swizzle, 8 rows 1024
// bytes apart).
__device__ __forceinline__ void mma_f8_wide(uint32_t d_tmem, uint32_t x, uint32_t w, uint32_t idesc,
                                            uint32_t accumulate) {
    constexpr uint32_t kHi = (1024 >> 4) | 1u << 14 | 2u << 29;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 dx, dw;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 dx, {%1, %5};\n\tmov.b64 dw, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], dx, dw, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(x), "r"(w), "r"(idesc), "r"(accumulate), "r"(kHi)
        : "memory");
}

__device__ __forceinline__ uint64_t twice(float s) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(s));
    return r;
}
struct QwTile {
    int e, wt;    // expert, weight tile
    int s0, cnt;  // first row of x, rows (1 to 128)
};

__device__ __forceinline__ QwTile qw_tile(const int *prefix, const int32_t *offsets, int E, int S, int u) {
    QwTile t;
    t.e = chunk_expert(prefix, E, u);
    const int lo = offsets ? offsets[t.e] : 0, hi = offsets ? offsets[t.e + 1] : S;
    const int runs = (hi - lo + 127) / 128, r = u - prefix[t.e];
    t.wt = r / runs;
    t.s0 = lo + (r - t.wt * runs) * 128;
    t.cnt = min(128, hi - t.s0);
    return t;
}

struct QwArgs {
    const int32_t *offsets;
    int E, S, n_in, n_out;
    const float *xs, *s0, *s1;  // scales of x [blocks, S], of w1 (or w), of v1
    void *out;                  // h8 or y
    float *out_scale;           // hs [blocks, S]
    unsigned *err;
};

template <bool UP, bool BF>
__global__ void __launch_bounds__(kQwThreads, 1)
k_quant_wide(const __grid_constant__ CUtensorMap tm_w0, const __grid_constant__ CUtensorMap tm_w1,
             const __grid_constant__ CUtensorMap tm_x, const QwArgs a) {
    using C = QwCfg<UP>;
    constexpr int kStages = C::kStages;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    QwHeader *hd = reinterpret_cast<QwHeader *>(smem + kStages * kQwStage + C::kOut);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nk = q_blocks(a.n_in), nblk = q_blocks(a.n_out);
    const int nwt = UP ? nblk : (nblk + 1) / 2;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(&hd->full[s], 1);
            ptx::mbar_init(&hd->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(&hd->tfull[b], 3);  // (the MMAs; the two warps with the scales)
            ptx::mbar_init(&hd->tempty[b], 8);
        }
        ptx::mbar_init(&hd->done, 1);
        ptx::fence_barrier_init();
        ptx::prefetch_tmap(&tm_w0);
        if (UP) ptx::prefetch_tmap(&tm_w1);
        ptx::prefetch_tmap(&tm_x);
    }
    if (warp == 1) tmem_alloc(&hd->tmem_base, 512);
    ptx::launch_dependents();
    // (the offsets are older than the launch ahead, which lets this one start behind its own
    // wait only, or is started so itself)
    if (warp == kQwEpilogue) q_tile_prefix(a.offsets, a.E, a.S, nwt, 128, hd->prefix, a.err);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = hd->tmem_base;
    const int n_units = hd->prefix[a.E], u0 = blockIdx.x, du = gridDim.x;

    if (warp < kQwEpilogue) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kQwRegsFeed));
        if (warp == 0) {
            // ------------------------------------------------------------ loads
            if (lane == 0) {
                // (both stay in L2: a weight tile serves the runs of its expert, x all weight tiles; with
                // normal priority for the weights 2048 rows of 8192 x 6144 took 99.3 us instead of 97.3)
                const uint64_t pol_w = ptx::policy_evict_last(), pol_x = ptx::policy_evict_last();
                auto weights = [&](const QwTile &t, uint32_t s, int kb) {
                    unsigned char *sp = smem + s * kQwStage + kQwTile;
                    uint64_t *fb = &hd->full[s];
                    ptx::mbar_arrive_expect_tx(fb, kQwStage);
                    tma_3d(sp, &tm_w0, kb * 128, t.wt * (UP ? 128 : 256), t.e, fb, pol_w);
                    tma_3d(sp + kQwTile, UP ? &tm_w1 : &tm_w0, kb * 128, UP ? t.wt * 128 : t.wt * 256 + 128, t.e,
                           fb, pol_w);
                };
                // the first stages' weights, which no kernel ahead writes, before the wait
                const uint32_t early = u0 < n_units ? min(kStages, nk) : 0;
                if (early) {
                    const QwTile t = qw_tile(hd->prefix, a.offsets, a.E, a.S, u0);
                    for (uint32_t k = 0; k < early; ++k) weights(t, k, k);
                }
                ptx::grid_dependency_wait();
                uint32_t it = 0;
                bool ok = true;
                for (int u = u0; ok && u < n_units; u += du) {
                    const QwTile t = qw_tile(hd->prefix, a.offsets, a.E, a.S, u);
                    for (int kb = 0; kb < nk; ++kb, ++it) {
                        const uint32_t s = it % kStages, ph = (it / kStages) & 1;
                        if (!(ok = wait_soon(&hd->empty[s], ph ^ 1, a.err))) break;
                        if (it >= early) weights(t, s, kb);
                        ptx::tma_load_2d(smem + s * kQwStage, &tm_x, kb * 128, t.s0, &hd->full[s], pol_x);
                    }
                }
                // copies in flight land before the block can end, and what the MMAs tell of its
                // last stages.  (Where a wait gave up, stages whose weights came early may
                // wait for rows that do not come: these waits end too.)
                it = max(it, early);
                for (uint32_t k = (it > kStages ? it - kStages : 0); k < it; ++k)
                    ptx::mbar_wait_hint(&hd->full[k % kStages], (k / kStages) & 1, a.err) &&
                        ptx::mbar_wait_hint(&hd->empty[k % kStages], (k / kStages) & 1, a.err);
            }
            __syncwarp();
        } else if (warp == 1) {
            // ------------------------------------------------------------ MMAs
            // (all lanes go along and one issues: in a branch of a single lane every MMA costs a
            // search for its operands' uniform registers)
            const bool one = elect_one();
            const int n = u0 < n_units ? ((n_units - 1 - u0) / du + 1) * nk : 0;
            const uint32_t base = (ptx::smem_u32(smem) & 0x3FFFFu) >> 4 | 1u << 16;
            uint32_t s = 0, ph = 0;
            bool ok = true;
#pragma unroll 1
            for (int it = 0; ok && it < n; ++it) {
                const uint32_t b = it & 1, bph = (it >> 1) & 1;
                ok = wait_soon(&hd->full[s], ph, a.err) && wait_soon(&hd->tempty[b], bph ^ 1, a.err);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t x = base + s * (kQwStage >> 4), w = x + (kQwTile >> 4);
                const uint32_t d = tmem + b * 256;
                if (one) {
                    mma_f8_wide(d, x, w, kQwIdesc, 0);
                    mma_f8_wide(d, x + 2, w + 2, kQwIdesc, 1);
                    mma_f8_wide(d, x + 4, w + 4, kQwIdesc, 1);
                    mma_f8_wide(d, x + 6, w + 6, kQwIdesc, 1);
                    mma_commit(&hd->tfull[b]);
                    mma_commit(&hd->empty[s]);
                }
                __syncwarp();
                if (++s == kStages) {
                    s = 0;
                    ph ^= 1;
                }
            }
            if (one) mma_commit(&hd->done);
            ptx::mbar_wait(&hd->done, 0, a.err);
            __syncwarp();
        } else {
            // ------------------------------------------------------------ scales
            // warps 2 and 3: 64 rows each.  A step's scales take the slot of the step four ago,
            // which the epilogue has read once the MMAs of the step two ago are done.
            ptx::grid_dependency_wait();
            const int r0 = (warp - 2) * 64 + lane;
            uint32_t it = 0;
            bool ok = true;
            for (int u = u0; ok && u < n_units; u += du) {
                const QwTile t = qw_tile(hd->prefix, a.offsets, a.E, a.S, u);
                const int row = min(t.s0 + r0, a.S - 1), blk = UP ? t.wt : t.wt * 2;
                const float *x0 = a.xs + row;
                const int x1 = min(t.s0 + r0 + 32, a.S - 1) - row, next = UP ? blk : min(blk + 1, nblk - 1);
                const float *w0 = a.s0 + ((size_t)t.e * nblk + blk) * nk;
                const float *w1 = (UP ? a.s1 : a.s0) + ((size_t)t.e * nblk + next) * nk;
                float v[4], more[4];  // of this k-block, of the next one
                auto fetch = [&](int kb) {
                    more[0] = x0[(size_t)kb * a.S];
                    more[1] = x0[(size_t)kb * a.S + x1];
                    more[2] = w0[kb];
                    more[3] = w1[kb];
                };
                fetch(0);
#pragma unroll 1
                for (int kb = 0; kb < nk; ++kb, ++it) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = more[j];
                    if (kb + 1 < nk) fetch(kb + 1);
                    if (it >= 2) ok = __all_sync(0xffffffffu, wait_soon(&hd->tfull[it & 1], ((it >> 1) - 1) & 1, a.err));
                    if (!ok) break;
                    hd->scale[it & 3][r0] = make_float2(v[0] * v[2], v[0] * v[3]);
                    hd->scale[it & 3][r0 + 32] = make_float2(v[1] * v[2], v[1] * v[3]);
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&hd->tfull[it & 1]);
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kQwRegsSums));
        // ------------------------------------------------------------ epilogue
        const int q = warp & 3, half = (warp - kQwEpilogue) >> 2;
        const uint32_t base0 = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)half * (UP ? 64 : 128);
        bool dead = false;  // a wait gave up: keep the barriers, skip the work
        ptx::grid_dependency_wait();  // (the result's last readers)
        uint32_t it = 0, tl = 0;
        for (int u = u0; u < n_units; u += du, ++tl) {
            const QwTile t = qw_tile(hd->prefix, a.offsets, a.E, a.S, u);
            const int r = q * 32 + lane;
            const bool mine = r < t.cnt;
            uint64_t acc[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = 0;
            for (int kb = 0; kb < nk; ++kb, ++it) {
                const uint32_t b = it & 1, bph = (it >> 1) & 1;
                if (!dead) dead = !__all_sync(0xffffffffu, wait_soon(&hd->tfull[b], bph, a.err));
                tc_fence_after();
                const uint32_t base = base0 + b * 256;
                if (!dead) {
                    const float2 f = hd->scale[it & 3][q * 32 + lane];
                    const uint64_t sc0 = twice(UP || half == 0 ? f.x : f.y), sc1 = UP ? twice(f.y) : sc0;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float v[32];
                        tmem_ld32(base + (c >> 1) * (UP ? 128 : 64) + (c & 1) * 32, v);
                        tmem_ld_wait();
                        if (c == 3) {  // the accumulator is read: the next MMAs may write it
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) ptx::mbar_arrive(&hd->tempty[b]);
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            fma2(acc[c * 16 + i], v[2 * i], v[2 * i + 1], c >> 1 ? sc1 : sc0);
                    }
                }
            }
            if (UP) {
                float h[64];
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const float2 x = both(acc[i]), y = both(acc[32 + i]);
                    h[2 * i] = q_silu(x.x) * y.x;
                    h[2 * i + 1] = q_silu(x.y) * y.y;
                    m = max(m, max(abs_bits(h[2 * i]), abs_bits(h[2 * i + 1])));
                }
                hd->amax[tl & 1][half][q * 32 + lane] = m;
                ptx::named_bar_sync(1 + q, 64);
                m = max(m, hd->amax[tl & 1][half ^ 1][q * 32 + lane]);
                float sc, inv;
                q_scale(m, sc, inv);
                if (mine && !dead) {
                    const int col = t.wt * 128 + half * 64;
                    uint8_t *hp = static_cast<uint8_t *>(a.out) + (size_t)(t.s0 + r) * a.n_out + col;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (col + 16 * i < a.n_out) {
                            const float *g = h + 16 * i;
                            *reinterpret_cast<uint4 *>(hp + 16 * i) =
                                make_uint4(q_pack4(g[0], g[1], g[2], g[3], inv),
                                           q_pack4(g[4], g[5], g[6], g[7], inv),
                                           q_pack4(g[8], g[9], g[10], g[11], inv),
                                           q_pack4(g[12], g[13], g[14], g[15], inv));
                        }
                    if (half == 0) a.out_scale[(size_t)t.wt * a.S + t.s0 + r] = sc;
                }
            } else {
                // 32 rows of 128 bytes at a time through shared memory, so that eight lanes
                // write a row's 128 bytes (16-byte chunks exchanged by the row: no conflicts)
                constexpr int kCols = BF ? 64 : 32, kSize = BF ? 2 : 4;
                uint8_t *buf = smem + kStages * kQwStage + (warp - kQwEpilogue) * 4096;
                const int row0 = q * 32, col0 = t.wt * 256 + half * 128;
                uint8_t *y = static_cast<uint8_t *>(a.out) + ((size_t)t.s0 * a.n_out + col0) * kSize;
                const int ch = lane & 7;
#pragma unroll
                for (int c = 0; c < 128 / kCols; ++c) {
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (BF) {
                                const float2 v = both(acc[c * 32 + 4 * i + j]);
                                const __nv_bfloat162 p = __floats2bfloat162_rn(v.x, v.y);
                                w[j] = *reinterpret_cast<const uint32_t *>(&p);
                            } else {
                                const float2 v = both(acc[c * 16 + 2 * i + (j >> 1)]);
                                w[j] = __float_as_uint(j & 1 ? v.y : v.x);
                            }
                        }
                        *reinterpret_cast<uint4 *>(buf + lane * 128 + ((i ^ (lane & 7)) << 4)) =
                            make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    __syncwarp();
                    const bool in = col0 + c * kCols + ch * (16 / kSize) < a.n_out && !dead;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int rr = i * 4 + (lane >> 3);
                        const uint4 w = *reinterpret_cast<const uint4 *>(buf + rr * 128 + ((ch ^ (rr & 7)) << 4));
                        if (in && row0 + rr < t.cnt)
                            *reinterpret_cast<uint4 *>(y + (size_t)(row0 + rr) * a.n_out * kSize + c * 128 +
                                                       ch * 16) = w;
                    }
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, 512);
}

template <bool UP, bool BF>
cudaError_t launch(const QuantGemm &g, const void *w0, const void *w1, QwArgs a, cudaStream_t st) {
    CUtensorMap mw0, mw1, mx;
    if (!q_weight_map(&mw0, w0, g.E, g.n_out, g.n_in) ||
        !q_weight_map(&mw1, UP ? w1 : w0, g.E, g.n_out, g.n_in) ||
        !q_row_map(&mx, g.x8, g.S, g.n_in, 128))
        return cudaErrorInvalidValue;
    const void *kern = (const void *)k_quant_wide<UP, BF>;
    static SmemOnce smem;
    cudaError_t e = smem.set(kern, QwCfg<UP>::kSmem);
    if (e != cudaSuccess) return e;
    a.offsets = g.offsets;
    a.E = g.E;
    a.S = g.S;
    a.n_in = g.n_in;
    a.n_out = g.n_out;
    a.xs = g.xs;
    a.err = device_info().err;
    void *args[] = {&mw0, &mw1, &mx, &a};
    LaunchScope ls(UP ? "quant_up_wide" : "quant_down_wide", st);
    return launch_pdl(kern, dim3(device_info().sm_count), dim3(kQwThreads), QwCfg<UP>::kSmem, st, args);
}

}  // namespace

cudaError_t launch_quant_wide_up(const QuantGemm &g, const QuantUp &u, cudaStream_t st) {
    QwArgs a{};
    a.s0 = u.s1;
    a.s1 = u.sv;
    a.out = u.h8;
    a.out_scale = u.hs;
    return launch<true, false>(g, u.w1, u.v1, a, st);
}

cudaError_t launch_quant_wide_down(const QuantGemm &g, const QuantDown &u, cudaStream_t st) {
    QwArgs a{};
    a.s0 = u.s;
    a.out = u.y;
    return u.y_bf16 ? launch<false, true>(g, u.w, nullptr, a, st)
                    : launch<false, false>(g, u.w, nullptr, a, st);
}

}  // namespace moe
