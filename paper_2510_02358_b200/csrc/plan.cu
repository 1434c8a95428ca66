// dsp_cache_plan: block tables, slots, positions and (for a beam tree) visibility bits of a step's
// tokens, from the requests' lengths.
//
// Everything a token needs follows from three prefix sums over the requests (tokens, blocks taken,
// blocks given back).  They are cheap (a few shuffles over at most 8192 numbers) against a grid-wide
// barrier or a second launch, so every CTA forms them for itself and then writes its share of the
// token rows and table entries: one launch, no workspace.  This needs the inputs to stay as they are
// while the call runs, which is why counts and ring position are outputs of their own; the block
// table and the ring are only written where no CTA reads (entries of blocks taken now are looked up
// in the ring, and a block given back goes behind the ring's tail).
//
// Bound by its latency: 8 requests of 17 tokens 4.8 us, 1024 of 32 (1.1 MB) 11.0 us, most of it what every CTA does for all requests: three
// passes that each load a request's numbers and divide (in 64 bits), and four scans with their barriers.
#include "dsp_common.cuh"

namespace dsp {
namespace {

struct PlanArgs {
    const int32_t *seq_len, *new_len, *count_in;
    const int64_t *ring_pos_in;
    int B, T, page, n_blocks, width;
    int32_t *table;
    long long table_stride;
    int32_t *ring;
    const int32_t *parent, *depth;
    int N;
    int32_t *count;
    int64_t *ring_pos;
    int32_t *cu, *kv_len;
    int64_t *slot;
    int32_t *position, *token_row;
    uint32_t *mask;
    int words;
    uint32_t *status;
};

// Exclusive prefix over the CTA's threads and the total (one value per thread).
__device__ __forceinline__ long long block_scan(long long v, long long *scratch, long long &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    long long incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += up;
    }
    __syncthreads();                                  // the scratch of the scan before has been read
    if (lane == 31) scratch[warp] = incl;
    __syncthreads();
    long long w = lane < warps ? scratch[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xFFFFFFFFu, w, o);
        if (lane >= o) w += up;
    }
    total = __shfl_sync(0xFFFFFFFFu, w, 31);
    const long long before = __shfl_sync(0xFFFFFFFFu, w, warp > 0 ? warp - 1 : 0);
    return (warp > 0 ? before : 0) + incl - v;
}

// Last index i in [0, n] with a[i] <= x, for a non-decreasing a with a[0] <= x.
__device__ __forceinline__ int last_not_above(const int32_t *a, int n, int x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

struct RowPlan {
    int seq, fresh, have;            // tokens cached and new (0 if the row brings none), blocks held
    long long need;
    uint32_t status;
    __device__ __forceinline__ RowPlan(const PlanArgs &a, int b) {
        seq = a.seq_len[b];
        fresh = a.new_len[b];
        have = a.count_in[b];
        status = 0u;
        if (seq < 0 || fresh < 0 || have < 0 || have > a.width || (a.parent && fresh > a.N + 1)) status = DSP_ROW_BAD_LENGTH;
        if ((long long)seq + fresh > 0x7FFFFFFF) status = DSP_ROW_BAD_LENGTH;
        need = ((long long)seq + fresh + a.page - 1) / a.page;
        if (!status && need > a.width) status = DSP_ROW_TABLE_FULL;
        if (status) fresh = 0;
    }
    __device__ __forceinline__ int lack() const { return status ? 0 : (int)max(need - have, 0LL); }
    __device__ __forceinline__ int surplus() const { return status ? 0 : (int)max(have - need, 0LL); }
};

__global__ void __launch_bounds__(1024) cache_plan_kernel(const PlanArgs a) {
    extern __shared__ int32_t s_rows[];
    int32_t *s_cu = s_rows, *s_take = s_cu + a.B + 1, *s_back = s_take + a.B + 1;     // exclusive prefixes
    int32_t *s_parent = s_back + a.B + 1;                                             // [N], trees only
    __shared__ long long s_scan[32];
    const int tid = threadIdx.x, per = (a.B + blockDim.x - 1) / blockDim.x;
    const int b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
    const long long head = a.ring_pos_in[0], tail = a.ring_pos_in[1];
    const long long free_blocks = max(0LL, min(tail - head, (long long)a.n_blocks));

    long long tokens = 0, lack = 0, sums = 0, back = 0, total;
    for (int b = b0; b < b1; ++b) tokens += RowPlan(a, b).fresh;
    const long long tokens0 = block_scan(tokens, s_scan, total);
    long long run = tokens0;
    for (int b = b0; b < b1; ++b) {
        RowPlan r(a, b);
        run += r.fresh;
        if (r.fresh > 0 && run > a.T) r.status |= DSP_ROW_PLAN_FULL;
        lack += r.lack();
    }
    const long long lack0 = block_scan(lack, s_scan, total);
    // the rows that are served: their tokens (low half) and blocks taken (high half), blocks given back
    for (int pass = 0; pass < 2; ++pass) {
        long long at = 0, at_back = 0;
        if (pass == 1) {
            at = block_scan(sums, s_scan, total);
            long long total_back;
            at_back = block_scan(back, s_scan, total_back);
            if (tid == 0) {
                s_cu[a.B] = (int32_t)(total & 0xFFFFFFFF);
                s_take[a.B] = (int32_t)(total >> 32);
                s_back[a.B] = (int32_t)total_back;
                if (blockIdx.x == 0) {
                    a.cu[a.B] = s_cu[a.B];
                    a.ring_pos[0] = head + s_take[a.B];
                    a.ring_pos[1] = tail + s_back[a.B];
                }
            }
        }
        run = tokens0;
        long long run_lack = lack0;
        for (int b = b0; b < b1; ++b) {
            RowPlan r(a, b);
            run += r.fresh;
            if (r.fresh > 0 && run > a.T) r.status |= DSP_ROW_PLAN_FULL;
            run_lack += r.lack();
            if (r.lack() > 0 && run_lack > free_blocks) r.status |= DSP_ROW_NO_BLOCKS;
            if (r.status) r.fresh = 0;
            const long long mine = (long long)r.lack() << 32 | r.fresh;
            if (pass == 0) {
                sums += mine;
                back += r.surplus();
                continue;
            }
            s_cu[b] = (int32_t)(at & 0xFFFFFFFF);
            s_take[b] = (int32_t)(at >> 32);
            s_back[b] = (int32_t)at_back;
            at += mine;
            at_back += r.surplus();
            if (blockIdx.x == 0) {
                a.cu[b] = s_cu[b];
                a.count[b] = min(max(r.have, 0), a.width) + r.lack() - r.surplus();
                a.kv_len[b] = max(r.seq, 0) + r.fresh;
                a.status[b] = r.status;
            }
        }
    }
    __syncthreads();

    const int n_tok = s_cu[a.B], n_take = s_take[a.B], n_back = s_back[a.B];
    const uint32_t nb = (uint32_t)a.n_blocks;
    // whatever the caller's counts say, entries stay inside the ring
    const uint32_t head_at = (uint32_t)((head % a.n_blocks + a.n_blocks) % a.n_blocks);
    const uint32_t tail_at = (uint32_t)((tail % a.n_blocks + a.n_blocks) % a.n_blocks);
    auto in_ring = [&](uint32_t at, uint32_t i) { return (at + i) % nb; };
    // block of the e-th table entry of row b (b brings tokens, so it is served)
    auto block_at = [&](int b, int e) {
        const int have = a.count_in[b];
        return e < have ? a.table[(long long)b * a.table_stride + e] : a.ring[in_ring(head_at, (uint32_t)(s_take[b] + e - have))];
    };
    const int stride = gridDim.x * blockDim.x, first = blockIdx.x * blockDim.x + tid;
    for (int i = first; i < n_take; i += stride) {
        const int b = last_not_above(s_take, a.B, i);
        const int e = a.count_in[b] + i - s_take[b];
        a.table[(long long)b * a.table_stride + e] = a.ring[in_ring(head_at, (uint32_t)i)];
    }
    for (int i = first; i < n_back; i += stride) {
        const int b = last_not_above(s_back, a.B, i);
        const int e = (int)(((long long)a.seq_len[b] + a.new_len[b] + a.page - 1) / a.page) + i - s_back[b];
        a.ring[in_ring(tail_at, (uint32_t)i)] = a.table[(long long)b * a.table_stride + e];
    }
    const bool tree = a.parent != nullptr;
    for (int t = first + (tree ? n_tok : 0); t < a.T; t += stride) {
        if (t >= n_tok) {
            a.slot[t] = -1;
            a.position[t] = -1;
            if (a.token_row) a.token_row[t] = -1;
            if (tree)
                for (int w = 0; w < a.words; ++w) a.mask[(long long)t * a.words + w] = 0u;
            continue;
        }
        const int b = last_not_above(s_cu, a.B, t);
        const int at = a.seq_len[b] + t - s_cu[b];
        const int e = at / a.page;
        a.slot[t] = (long long)block_at(b, e) * a.page + (at - e * a.page);
        a.position[t] = at;
        if (a.token_row) a.token_row[t] = b;
    }
    if (!tree) return;
    // a CTA takes whole rows: the tree's parents sit in shared memory, one thread per token and mask
    // word follows the path to the root (parents are earlier nodes, so every path ends)
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        const int t0 = s_cu[b], n = s_cu[b + 1] - t0;
        if (n == 0) continue;                                      // uniform over the CTA
        __syncthreads();
        for (int i = tid; i < n - 1; i += blockDim.x) {
            const int p = a.parent[(long long)b * a.N + i];
            s_parent[i] = p >= 0 && p < i ? p : -1;
        }
        __syncthreads();
        for (int i = tid; i < n * a.words; i += blockDim.x) {
            const int tok = i / a.words, w = i - tok * a.words;
            uint32_t bits = w == 0 ? 1u : 0u;
            for (int node = tok - 1; node >= 0; node = s_parent[node]) {
                const int j = node + 1 - 32 * w;
                if (j < 0) break;                                  // the rest of the path lies in earlier words
                if (j < 32) bits |= 1u << j;
            }
            a.mask[(long long)(t0 + tok) * a.words + w] = bits;
        }
        const int seq = a.seq_len[b];
        for (int i = tid; i < n; i += blockDim.x) {
            const int at = seq + i, e = at / a.page;
            a.slot[t0 + i] = (long long)block_at(b, e) * a.page + (at - e * a.page);
            a.position[t0 + i] = i == 0 ? seq : seq + 1 + a.depth[(long long)b * a.N + i - 1];
            if (a.token_row) a.token_row[t0 + i] = b;
        }
    }
}

}  // namespace
}  // namespace dsp

extern "C" int32_t dsp_cache_plan(const int32_t *seq_len, const int32_t *new_len, const int32_t *block_count_in,
                                  const int64_t *ring_pos_in, int32_t B, int32_t T, int32_t page_size,
                                  int32_t n_blocks, int32_t max_blocks,
                                  int32_t *block_table, int64_t table_stride, int32_t *free_ring,
                                  const int32_t *node_parent, const int32_t *node_depth, int32_t N,
                                  int32_t *block_count, int64_t *ring_pos, int32_t *cu_new, int32_t *kv_len,
                                  int64_t *slot, int32_t *position, int32_t *token_row,
                                  uint32_t *mask, int32_t mask_words, uint32_t *row_status, dsp_stream_t stream) {
    using namespace dsp;
    const bool tree = node_parent || node_depth;
    if (B < 0 || T < 0 || page_size < 1 || n_blocks < 1 || max_blocks < 1 || table_stride < max_blocks) return DSP_ERR_INVALID_ARG;
    if (tree && (!node_parent || !node_depth || N < 1 || (T > 0 && !mask) || (long long)mask_words * 32 < (long long)N + 1))
        return DSP_ERR_INVALID_ARG;
    if (B > DSP_MAX_PLAN_ROWS || (tree && N + 1 > DSP_MAX_L)) return DSP_ERR_UNSUPPORTED;
    if (B == 0 && T == 0) return DSP_OK;
    if (!ring_pos_in || !ring_pos || !cu_new || !free_ring || (T > 0 && (!slot || !position))) return DSP_ERR_INVALID_ARG;
    if (B > 0 && (!seq_len || !new_len || !block_count_in || !block_table || !block_count || !kv_len || !row_status))
        return DSP_ERR_INVALID_ARG;
    if (ring_pos == ring_pos_in || block_count == block_count_in) return DSP_ERR_INVALID_ARG;
    PlanArgs a = {};
    a.seq_len = seq_len; a.new_len = new_len; a.count_in = block_count_in; a.ring_pos_in = ring_pos_in;
    a.B = B; a.T = T; a.page = page_size; a.n_blocks = n_blocks; a.width = max_blocks;
    a.table = block_table; a.table_stride = table_stride; a.ring = free_ring;
    a.parent = node_parent; a.depth = node_depth; a.N = tree ? N : 0;
    a.count = block_count; a.ring_pos = ring_pos; a.cu = cu_new; a.kv_len = kv_len;
    a.slot = slot; a.position = position; a.token_row = token_row;
    a.mask = mask; a.words = mask_words; a.status = row_status;
    // a request's lengths are scanned by every CTA: few threads have the short barrier (1024 requests of 32 new tokens: 11.0 us with
    // 256 threads, 12.4 with 1024), many the short loop (4096 requests of 8: 44 and 21 us)
    const unsigned threads = B <= 1024 ? 256u : 1024u;
    const size_t smem = ((size_t)3 * (B + 1) + a.N) * sizeof(int32_t);
    if (smem > 40 * 1024)
        DSP_CUDA_TRY(cudaFuncSetAttribute(cache_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                          (int)(((size_t)3 * (DSP_MAX_PLAN_ROWS + 1) + DSP_MAX_L) * sizeof(int32_t))));
    long long grid = tree ? B : ((long long)T + 4 * threads - 1) / (4 * threads);
    grid = grid < 1 ? 1 : grid > 148 ? 148 : grid;
    cache_plan_kernel<<<(unsigned)grid, threads, smem, reinterpret_cast<cudaStream_t>(stream)>>>(a);
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}
