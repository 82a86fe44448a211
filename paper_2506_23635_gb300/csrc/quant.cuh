// 8-bit experts: what their kernels share.  Numbers are e4m3; a scale (fp32) belongs to
// each 128 numbers of an activation row and to each 128 x 128 block of a weight matrix.
#pragma once

#include <stdint.h>

#include "paged.cuh"  // (e4m3 conversions, SmemOnce)
#include "tc.cuh"

namespace moe {

constexpr int kQBlock = 128;    // numbers that share a scale, along a row
constexpr int kQMinExp = -100;  // the quantisers' scales are at least 2^-100
constexpr int kQMaxCtas = 160;  // of the streaming kernel, one for each SM

__host__ __device__ inline int q_blocks(int n) { return (n + kQBlock - 1) / kQBlock; }

// The scale of a block whose largest magnitude has these bits: the smallest power
// of two that holds it (448 = 1.75 2^8), and its reciprocal; NaN where the block has a
// value that is not finite.
__device__ __forceinline__ void q_scale(uint32_t amax_bits, float &scale, float &inv) {
    if (amax_bits >= 0x7f800000u) {
        scale = inv = __uint_as_float(0x7fffffffu);
        return;
    }
    const int e = max((int)(amax_bits >> 23) - 127 - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0),
                      kQMinExp);
    scale = __uint_as_float((uint32_t)(e + 127) << 23);
    inv = __uint_as_float((uint32_t)(127 - e) << 23);
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// SiLU by the fast exponential and quotient: off by at most (|a| + 8) 2^-23 of itself (and half
// a step of the smallest numbers), far below the e4m3 rounding that follows (with expf and a full
// division the experts of 2048 tokens took 5%, 300 tokens of 40 small experts 25% longer).
// exp(-|a|), so that the divisor stays within 2: the fast quotient is 0 for divisors beyond 2^126.
__device__ __forceinline__ float q_silu(float a) {
    const float e = __expf(-fabsf(a));
    return __fdividef(a < 0.f ? a * e : a, 1.f + e);
}

// Four values times inv (a power of two: exact but for numbers far below the
// block's smallest e4m3) rounded to e4m3, the first in the low byte.
__device__ __forceinline__ uint32_t q_pack4(float a, float b, float c, float d, float inv) {
    return e4m3x2(a * inv, b * inv) | e4m3x2(c * inv, d * inv) << 16;
}

// 16 consecutive fp32 columns of this warp's 32 tensor-memory lanes.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&v)[16]) {
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

__device__ __forceinline__ void tma_3d(void *dst, const CUtensorMap *m, int32_t x, int32_t y,
                                       int32_t z, uint64_t *bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        ".L2::cache_hint [%0], [%1, {%2, %3, %4}], [%5], %6;" ::"r"(ptx::smem_u32(dst)),
        "l"(m), "r"(x), "r"(y), "r"(z), "r"(ptx::smem_u32(bar)), "l"(policy)
        : "memory");
}

// A wait that is over soon: the clock is looked at after 256 tries only.
__device__ __forceinline__ bool wait_soon(uint64_t *bar, uint32_t parity, unsigned *err) {
    uint64_t t0 = 0;
    for (uint32_t it = 1;; ++it) {
        if (ptx::mbar_try_wait(bar, parity)) return true;
        if ((it & 255u) == 0) {
            const uint64_t now = ptx::globaltimer();
            if (t0 == 0) t0 = now;
            if (now - t0 > ptx::kWaitLimitNs) {
                set_error(err, kErrTimeout);
                return false;
            }
        }
    }
}

// One lane of the warp, always the same.
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r));
    return r != 0;
}

// Two fp32 at once: acc += v * s.
__device__ __forceinline__ void fma2(uint64_t &acc, float v0, float v1, uint64_t s) {
    asm("{\n\t.reg .b64 v;\n\tmov.b64 v, {%1, %2};\n\tfma.rn.f32x2 %0, v, %3, %0;\n\t}"
        : "+l"(acc)
        : "f"(v0), "f"(v1), "l"(s));
}
__device__ __forceinline__ float2 both(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}

// prefix[e]: tiles of the experts ahead of e, nwt for each run of `rows` rows (one warp).
__device__ __forceinline__ void q_tile_prefix(const int32_t *offsets, int E, int S, int nwt, int rows,
                                              int *prefix, unsigned *err) {
    const int lane = threadIdx.x & 31;
    int run = 0;
    for (int base = 0; base < E; base += 32) {
        const int e = base + lane;
        int c = 0;
        if (e < E) {
            const int lo = offsets ? offsets[e] : 0, hi = offsets ? offsets[e + 1] : S;
            if (lo < 0 || hi < lo || hi > S) set_error(err, kErrIndex);
            else c = ((hi - lo + rows - 1) / rows) * nwt;
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

// A grouped product of 8-bit operands: rows x8 [S, n_in] in groups given by offsets
// [E+1] (null: one group of S rows) times each group's matrix w8 [E, n_out, n_in].
struct QuantGemm {
    int E, S, n_in, n_out;
    const int32_t *offsets;
    const void *x8;
    const float *xs;  // [q_blocks(n_in), S]: the rows' scales of one k-block side by side
};

// What the streaming kernel (quant_stream_tc.cu) needs beside its operands: slots
// for tiles that several CTAs share, and a counter for each CTA, zero at the start.
struct QuantParts {
    float *part;
    int *count;
};
// Rows of x8 that a tile of the streaming kernel takes: half as many again as the
// groups have on average (64 tokens of 4 experts of 16: 32), one group's own number.
inline int q_stream_cols(int E, long long S) {
    const long long rows = E == 1 ? S : (3 * S + 2 * E - 1) / (2 * E);
    return rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
}
inline size_t q_part_floats(int cols, bool up) {
    return (size_t)2 * kQMaxCtas * 128 * cols * (up ? 2 : 1);
}

// up: h8, hs = quantised SiLU(x.w1) (x.v1); else y (fp32 or bf16) = x.w
struct QuantUp {
    const void *w1, *v1;
    const float *s1, *sv;
    void *h8;
    float *hs;  // [q_blocks(n_out), S]
};
struct QuantDown {
    const void *w;
    const float *s;
    void *y;
    int y_bf16;
};
cudaError_t launch_quant_stream_up(const QuantGemm &g, const QuantUp &u, const QuantParts &p,
                                   int cols, cudaStream_t st);
// alone: not behind the up projection, whose CTAs it shares the SMs with otherwise.  The
// launch ahead lets either start behind its own wait only (the offsets and weights are read
// before this kernel's).
cudaError_t launch_quant_stream_down(const QuantGemm &g, const QuantDown &u, const QuantParts &p,
                                     int cols, bool alone, cudaStream_t st);

// The same for many rows a group (quant_wide_tc.cu); it, too, reads offsets and weights early.
cudaError_t launch_quant_wide_up(const QuantGemm &g, const QuantUp &u, cudaStream_t st);
cudaError_t launch_quant_wide_down(const QuantGemm &g, const QuantDown &u, cudaStream_t st);

// 8-bit weights [n, rows, cols]: boxes of 128 x 128, zeros outside each matrix.
inline bool q_weight_map(CUtensorMap *m, const void *base, uint64_t n, uint64_t rows,
                         uint64_t cols) {
    auto fn = tc::encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {cols, rows, n};
    cuuint64_t strides[2] = {cols, rows * cols};
    cuuint32_t box[3] = {128u, 128u, 1u};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void *>(base), dims, strides, box,
              estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// 8-bit rows [rows, cols]: boxes of box_rows x 128, zeros outside.
inline bool q_row_map(CUtensorMap *m, const void *base, uint64_t rows, uint64_t cols,
                      uint32_t box_rows) {
    auto fn = tc::encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {cols};
    cuuint32_t box[2] = {128u, box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box,
              estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace moe
