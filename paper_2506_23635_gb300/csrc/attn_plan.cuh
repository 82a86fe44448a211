// The plan of an attention call, made on the device: which of its tokens the
// prefill attention takes in tiles and which are attended one by one.
#pragma once

#include "ptx.cuh"

namespace moe {

constexpr int kMaxSaTokens = 65536;

// What the attention's plan is made from, and where it goes (plan.head null:
// the call needs none).
struct PlanArgs {
    const int32_t *seq, *pos;
    int n_seq, L;
    AttnPlan plan;
};

// The plan of an attention call, by one block of NT threads.  A run is the
// longest stretch of tokens that are consecutive positions of one sequence;
// its tiles are cut from its first token on.  Tiles of at least
// MIN_ROWS tokens are listed by falling length (a counting sort over
// their key/value tiles; tiles of the same length in any order: no result
// depends on it), the tokens of the others in ascending order.  Run starts are
// kept as one bit a token.  It runs beside the pre-norm's other blocks and is
// done before the projection after them ends.
constexpr int kPlanBins = 256;

// Returns the number of tokens left, in every thread.
template <int NT, int MIN_ROWS = kAttnTileMinRows>
__device__ int plan_attention(int T, const PlanArgs &a) {
    static_assert(NT >= kPlanBins && NT % 32 == 0 && NT <= 1024, "a thread for each bin, a lane a warp");
    __shared__ uint32_t brk[kMaxSaTokens / 32];  // bit t: a run starts at token t
    __shared__ int last[kMaxSaTokens / 32];      // the last run start ahead of each word
    __shared__ int bins[kPlanBins];
    __shared__ int wsum[NT / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int nw = (T + 31) / 32;
    for (int t = tid; t < nw * 32; t += NT) {
        bool b = false;
        if (t < T) {
            const int sq = a.seq[t], p = a.pos[t];
            // (a token outside the cache is a run of its own)
            b = t == 0 || sq < 0 || sq >= a.n_seq || p <= 0 || p >= a.L || a.seq[t - 1] != sq ||
                a.pos[t - 1] != p - 1;
        }
        const uint32_t m = __ballot_sync(0xffffffffu, b);
        if (lane == 0) brk[t >> 5] = m;
    }
    if (tid < kPlanBins) bins[tid] = 0;
    __syncthreads();
    if (warp == 0) {
        int run = 0;
        for (int w0 = 0; w0 < nw; w0 += 32) {
            const int w = w0 + lane;
            int v = w < nw && brk[w] ? w * 32 + 31 - __clz(brk[w]) : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v = max(v, u);
            }
            v = max(v, run);
            const int ahead = __shfl_up_sync(0xffffffffu, v, 1);
            if (w < nw) last[w] = lane == 0 ? run : ahead;
            run = __shfl_sync(0xffffffffu, v, 31);
        }
    }
    __syncthreads();
    // the tile of token t: its first token, and its tokens
    auto tile_of = [&](int t, int &ts, int &rows) {
        const uint32_t m = brk[t >> 5] & (0xffffffffu >> (31 - (t & 31)));
        const int rs = m ? (t & ~31) + 31 - __clz(m) : last[t >> 5];
        ts = rs + ((t - rs) & ~(kAttnTile - 1));
        int end = min(ts + kAttnTile, T);
        int w = (ts + 1) >> 5;
        uint32_t n = w < nw ? brk[w] & (0xffffffffu << ((ts + 1) & 31)) : 0u;
        while (n == 0 && (w + 1) * 32 < end) n = brk[++w];
        if (n) end = min(end, w * 32 + __ffs(n) - 1);
        rows = end - ts;
    };
    auto bin_of = [&](int ts, int rows) {  // falling length
        return kPlanBins - 1 - min(kPlanBins - 1, (a.pos[ts] + rows - 1) / kAttnTile);
    };
    int n_left = 0;
    for (int t0 = 0; t0 < T; t0 += NT) {
        const int t = t0 + tid;
        bool left = false;
        if (t < T) {
            int ts, rows;
            tile_of(t, ts, rows);
            left = rows < MIN_ROWS;
            if (!left && t == ts) atomicAdd(&bins[bin_of(ts, rows)], 1);
        }
        const uint32_t m = __ballot_sync(0xffffffffu, left);
        if (lane == 0) wsum[warp] = __popc(m);
        __syncthreads();
        int at = n_left + __popc(m & ((1u << lane) - 1u));
        const int c = lane < NT / 32 ? wsum[lane] : 0;
        at += __reduce_add_sync(0xffffffffu, lane < warp ? c : 0);
        n_left += __reduce_add_sync(0xffffffffu, c);
        if (left) a.plan.left[at] = t;
        __syncthreads();
    }
    if (warp == 0) {  // bins -> first place of each, a lane a few in a row
        constexpr int B = kPlanBins / 32;
        int c[B], v = 0;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            c[b] = bins[lane * B + b];
            v += c[b];
        }
        const int mine = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        if (lane == 31) *a.plan.head = AttnPlanHead{v, n_left, 0, 0};
        v -= mine;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            bins[lane * B + b] = v;
            v += c[b];
        }
    }
    __syncthreads();
    for (int t = tid; t < T; t += NT) {
        int ts, rows;
        tile_of(t, ts, rows);
        if (t == ts && rows >= MIN_ROWS)
            a.plan.tiles[atomicAdd(&bins[bin_of(ts, rows)], 1)] =
                make_int4(ts, rows, a.pos[ts], a.seq[ts]);
    }
    return n_left;
}

}  // namespace moe
