// The paged 8-bit key/value cache: what its kernels share (paged.cu).
#pragma once

#include <stdint.h>

#include <atomic>

#include "tc.cuh"

namespace moe {

constexpr int kPagedDh = 128;        // head_dim
constexpr int kPagedMaxGroup = 8;    // query heads per key/value head
constexpr int kPagedMinExp = -100;   // scales are at least 2^-100

// Where the positions of the sequences lie: page_table [n_seq, max_pages].
struct PageView {
    const int32_t *table;
    int n_seq, max_pages, n_pages;
    int shift;  // log2(page_size)

    // token (sequence sq, position p) lies inside the table
    __device__ __forceinline__ bool inside(int sq, int p) const {
        return sq >= 0 && sq < n_seq && p >= 0 && (p >> shift) < max_pages;
    }
    // page of the sequence's page index i, or -1 where the table holds none
    __device__ __forceinline__ int page(int sq, int i) const {
        const int pg = table[(size_t)sq * max_pages + i];
        return pg >= 0 && pg < n_pages ? pg : -1;
    }
};

// Two floats -> two e4m3 (round to nearest even, largest magnitude 448; NaN
// stays NaN), the first in the low byte; and back to two halves (exact).
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t v) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)v));
    return r;
}
__device__ __forceinline__ float2 e4m3x2_to_float2(uint32_t v) {
    const uint32_t h = e4m3x2_to_f16x2(v);
    float2 f;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}"
        : "=f"(f.x), "=f"(f.y)
        : "r"(h));
    return f;
}

// A kernel's dynamic shared memory, asked for once per device.
struct SmemOnce {
    std::atomic<uint64_t> done{0};  // bit: device
    cudaError_t set(const void *kern, size_t bytes) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const uint64_t bit = dev < 64 ? 1ull << dev : 0;
        if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
        return e;
    }
};

// The tokens that the decode attention takes one by one, made on the device
// (k_paged_plan): list[i] is a token, before[i] the position tiles (of
// kPagedTile positions; none for a token outside the table) of the list's tokens
// ahead of it, entry n_list those of all.  released: n_list + 1, stored with release
// semantics once all of it is (zero before): who acquires that sees the list and
// whatever was complete ahead of the plan.  count: counters of finished parts, two
// for each CTA, zero at the start.
constexpr int kPagedSmall = 128;  // tokens of a call that needs no list, at most
constexpr int kPagedTile = 128;
constexpr int kPagedMaxCtas = 320;
struct PagedList {
    int *n_list, *released;
    int *list;
    long long *before;
    int *count;
};
// a part's slot in the workspace: 8 rows of 128 sums, 8 pairs (base, sum); two
// slots for each CTA
constexpr int kPagedSlot = kPagedMaxGroup * (kPagedDh + 2);
constexpr size_t kPagedPartFloats = (size_t)2 * kPagedMaxCtas * kPagedSlot;

struct PagedAttn {
    int T, Hq, Hkv, page_size;
    PageView pv;
    const int32_t *seq, *pos;
    const void *q, *kp, *vp;
    const float *ks, *vs;
    void *ctx;
};
// A page's rows of one head as a box: 8-bit [rows, 128].
inline bool paged_map(CUtensorMap *m, const void *base, const PagedAttn &a, bool swizzle128) {
    auto fn = tc::encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {kPagedDh, (cuuint64_t)a.pv.n_pages * a.Hkv * a.page_size};
    cuuint64_t strides[1] = {kPagedDh};
    cuuint32_t box[2] = {kPagedDh, (cuuint32_t)a.page_size};
    cuuint32_t estr[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box,
              estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              swizzle128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Fewer consecutive tokens than this are attended one by one: a tile costs the same
// whatever its rows (24 chunks at position 2000, DBRX's heads: 151 us; one by one 196
// for 16 tokens each, 244 for 20; four at position 3000: 55 and 61 for 16, so that 12
// to 14 break even).
constexpr int kPagedTileMinRows = 16;

// Attention of the plan's tiles (paged_prefill_tc.cu).  part, count: where a unit
// of work is shared by several CTAs; 2 counters a part, zero at the start.
constexpr int kPagedUnitParts = 160;  // one for each SM
constexpr size_t kPagedUnitPartFloats = (size_t)kPagedUnitParts * 2 * 128 * (128 + 2);
cudaError_t launch_paged_prefill_tc(const PagedAttn &a, const AttnPlan &plan, float *part,
                                    int *count, cudaStream_t st);
// Attention of single tokens (paged_decode_tc.cu).  small: up to kPagedSmall tokens,
// all taken one by one, right behind k_paged_plan: the kernel lists them itself, and only
// the counters are the plan's.  Otherwise of the listed tokens, behind the prefill
// attention, whose results are not read here: this kernel runs beside it, as that
// one leaves SMs, on what the plan has released.
cudaError_t launch_paged_decode_tc(const PagedAttn &a, const PagedList &l, float *part, bool small,
                                   cudaStream_t st);


// ---- host side (paged.cu), for the attention block over the paged cache --------

// What the shape and the call's pointers have to be.
moe_status check_paged(const moe_sa_dims *d, const moe_paged_dims *pd);
moe_status check_paged_call(const moe_sa_dims *d, const moe_paged_dims *pd, int32_t T,
                            const int32_t *seq, const int32_t *pos, const int32_t *table,
                            const void *kp, const void *vp, const float *ks, const float *vs);
// moe_paged_append of an fp32 projection in n_part parts (0: as `split` says).
cudaError_t launch_paged_append(const moe_sa_dims &d, const moe_paged_dims &pd, int T,
                                const float *qkv, int n_part, long long part_stride,
                                const ProjSplit &split, const int32_t *seq, const int32_t *pos,
                                const int32_t *table, void *q, void *kp, void *vp, float *ks,
                                float *vs, cudaStream_t st);
cudaError_t launch_paged_attend(const moe_sa_dims &d, const moe_paged_dims &pd, int T,
                                const void *q, const int32_t *seq, const int32_t *pos,
                                const int32_t *table, const void *kp, const void *vp,
                                const float *ks, const float *vs, void *ctx, void *ws,
                                cudaStream_t st);

}  // namespace moe
