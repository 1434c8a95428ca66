// What the kernels of dsp_attn_kv4 share: their arguments, the cut of the work over CTAs, and the
// workspace of partial results.
#pragma once

#include "kv4.cuh"

namespace dsp {

struct AttnArgs {
    const __nv_bfloat16 *q;
    long long q_t, q_h;
    int B, T, Hq, Hkv, group;                    // group: query heads per key head
    const uint8_t *cache;
    int n_blocks, page;
    const int32_t *table;
    long long table_stride;
    int max_blocks;
    const int32_t *kv_len, *cu;
    int max_new;
    float scale_log2;                            // scale * log2(e): scores are formed in base 2
    int mask_kind;
    const uint32_t *bits;
    int words;
    __nv_bfloat16 *out;
    // workspace
    struct SplitUnit *split;                     // [grid] the unit that starts in a CTA's share and ends in a later one's
    float *part;                                 // [grid][2] partial results
};

// Work is cut along the cache, so that few long requests fill the GPU as well as many short ones.
// A unit is one tile of query rows (query i, head hh of the group: row i * group + hh) of one request
// and key head; it is as many steps long as its part of the cache has tiles of tokens.  All units' steps
// lie on one line, and CTA w takes an equal share of it.  A unit inside one share is finished there; of
// one that crosses shares each CTA leaves a partial result, joined by a second, small kernel.
struct SplitUnit {
    int b, h, tile, last_cta;                    // last_cta < 0: none
};

// A request's place on that line.
struct Request {
    int b, n_new, kv, rows;                      // new tokens, tokens in all (may be fewer), query rows per key head
    int row0;                                    // first row of q
    int tiles, steps;                            // query tiles, steps of each unit
    __device__ __forceinline__ void load(const AttnArgs &a, int b_, int tile_rows, int step_tokens) {
        b = b_;
        row0 = max(a.cu[b], 0);
        n_new = max(a.cu[b + 1] - row0, 0);
        kv = (int)max(0LL, min((long long)a.kv_len[b], min((long long)a.max_blocks * a.page, 0x7FFFFF00LL)));
        rows = max(min(min(n_new, a.T - row0), a.max_new), 0) * a.group;      // of the tokens that the call answers
        tiles = (rows + tile_rows - 1) / tile_rows;
        steps = max(1, (kv + step_tokens - 1) / step_tokens);
    }
    __device__ __forceinline__ long long length(int Hkv) const { return (long long)Hkv * tiles * steps; }
};

__device__ __forceinline__ long long share_begin(long long total, int cta, int ctas) { return total * cta / ctas; }
// CTA whose share holds place x of the line.
__device__ __forceinline__ int cta_of(long long x, long long total, int ctas) { return (int)(((x + 1) * ctas - 1) / total); }

// Where the line is entered: request, and the step within the request, at which the CTA's share begins.
struct LineStart {
    long long total, begin, end;                 // of the line; this CTA's share
    int ctas;                                    // CTAs with a share: none is empty
    int b;
    long long before;                            // line place where request b begins
};
// Every thread of the CTA calls it; scratch: 32 long longs and the result's place in shared memory.
// min_share: no CTA's share is shorter.
template <typename Req>
__device__ __forceinline__ void enter_line(const AttnArgs &a, int tile_rows, int step_tokens, int min_share, long long *scratch, LineStart *out) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int per = (a.B + blockDim.x - 1) / blockDim.x;
    const int b0 = min((int)threadIdx.x * per, a.B), b1 = min(b0 + per, a.B);
    long long mine = 0;
    for (int b = b0; b < b1; ++b) {
        Req r;
        r.load(a, b, tile_rows, step_tokens);
        mine += r.length(a.Hkv);
    }
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += up;
    }
    if (lane == 31) scratch[warp] = incl;
    __syncthreads();
    long long before = incl - mine, total = 0;
    for (int w = 0; w < warps; ++w) {
        const long long v = scratch[w];
        total += v;
        if (w < warp) before += v;
    }
    const int ctas = (int)min((long long)gridDim.x, total > 0 ? max(1LL, total / min_share) : 0LL);
    const bool idle = (int)blockIdx.x >= ctas;
    const long long begin = idle ? total : share_begin(total, blockIdx.x, ctas), end = idle ? total : share_begin(total, blockIdx.x + 1, ctas);
    if (begin >= before && begin < before + mine) {
        for (int b = b0; b < b1; ++b) {
            Req r;
            r.load(a, b, tile_rows, step_tokens);
            const long long n = r.length(a.Hkv);
            if (begin < before + n) {
                out->b = b;
                out->before = before;
                break;
            }
            before += n;
        }
    }
    if (threadIdx.x == 0) {
        out->total = total;
        out->begin = begin;
        out->end = end;
        out->ctas = ctas;
    }
    __syncthreads();
}

}  // namespace dsp
